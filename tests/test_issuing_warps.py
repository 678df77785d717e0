"""Warps of the operators over pages in which one lane issues the products: a rule that can be checked in their source (no GPU)."""
import os
import re

from tests.test_kernel_source import CSRC, _calls


def test_waits_of_the_operators_over_pages():
    """Every wait's answer is the warp's, as in the kernels whose leader is named by an assignment: a lane left behind for two phases would wait for a parity that is not coming."""
    seen = {}
    for name in ("esp_paged_tc.cu", "esp_key_weights_tc.cu"):
        text = open(os.path.join(CSRC, name)).read()
        for m in re.finditer(r"\{elect_lane\(\)\};", text):
            role = text[m.end():text.index("\n    } else", m.end())]
            together = list(_calls(role, "__all_sync"))
            waits = list(_calls(role, "mbar_wait"))
            assert all(any(b < beg and end <= e for b, e in together) for beg, end in waits), name
            seen[name] = seen.get(name, 0) + len(waits)
    assert min(seen.get("esp_paged_tc.cu", 0), seen.get("esp_key_weights_tc.cu", 0)) >= 2, seen
