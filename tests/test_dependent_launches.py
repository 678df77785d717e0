"""Kernels that may start while the one in front of them still runs (programmatic dependent launch): a rule that can be checked in their source (no GPU)."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_17942_b200", "csrc")


def _block(text, start):
    """End of the braces that open at or behind `start`."""
    i = text.index("{", start) + 1
    depth = 1
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return i


def _kernels():
    """(file, name, body) of every kernel, without comments and without the lambdas in it, whose returns are not the kernel's."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)
        for m in re.finditer(r"__global__[^;{]*?\b(k_\w+)\s*\(", text):
            body = text[text.index("{", m.end()):_block(text, m.end())]
            while True:
                inner = re.search(r"= \[&?\]\([^{;]*\)[^{;]*\{", body)
                if not inner:
                    break
                body = body[:inner.start()] + body[_block(body, inner.start()):]
            yield os.path.basename(path), m.group(1), body


def test_a_dependent_kernel_waits_on_every_path():
    """Who comes behind such a kernel is ordered behind it alone, so it must not end before its predecessor has: no return in front of its first wait."""
    seen = set()
    for name, kernel, body in _kernels():
        wait = body.find("pdl_wait()")
        if wait < 0:
            continue
        seen.add(kernel)
        for m in re.finditer(r"\breturn\b", body[:wait]):
            raise AssertionError(f"{name}: {kernel} can end without waiting: {body[max(0, m.start() - 80):m.end()]}")
    assert {"k_key_weights_join", "k_evict_move", "k_sample_list", "k_sample_rest", "k_paged_merge", "k_paged_merge_few"} <= seen
