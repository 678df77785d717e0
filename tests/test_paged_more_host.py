"""Weights of cached positions, eviction, sampling and acceptance as far as they go without a GPU: structs of the binding and refusals of the C entry points (nothing is launched)."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_paged_host import ARG, BADCFG, ROOT, WORKSPACE, X, _batch, _cache, _heads, lib  # noqa: F401

BIG = 1 << 40


def _ref(x):
    return None if x is None else ctypes.byref(x)


def test_structs_mirror_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "esp.h")).read(), flags=re.S)
    for cname, ctype in (("esp_paged_slots", P.esp_paged_slots), ("esp_sampling", P.esp_sampling)):
        end = text.index("} %s;" % cname)
        body = text[text.rindex("typedef struct {", 0, end) + len("typedef struct {"):end]
        members = [n.strip().lstrip("*").strip() for d in body.split(";") if d.strip()
                   for n in re.sub(r"^(const\s+)?\w+\s*\*?", "", d.strip(), count=1).split(",")]
        assert members == [f[0] for f in ctype._fields_], cname


def _slots(data=5 * X, page=32, token=1, head=16):
    return P.esp_paged_slots(data, page, token, head)


def _weights(lib, tokens=4, cache=None, batch=None, q=None, lse=X, anc=None, window=0, scale=0.0, last=0, keep=1.0, scores=None, scratch=X, nbytes=1 << 40):  # noqa: F811
    return lib.esp_paged_key_weights(tokens, _ref(cache or _cache()), _ref(batch or _batch()), _ref(q or _heads(n=4)), lse, anc, window, scale, last, keep, _ref(scores or _slots()), scratch,
                                     nbytes, None)


def test_key_weights_refusals(lib):  # noqa: F811
    bad = [(ARG, dict(tokens=-1)), (ARG, dict(tokens=2 ** 30 + 1)), (ARG, dict(lse=None)), (ARG, dict(lse=X + 2)), (ARG, dict(window=-1)), (ARG, dict(last=-1)), (ARG, dict(scale=-1.0)),
           (ARG, dict(scale=math.nan)), (ARG, dict(keep=-0.5)), (ARG, dict(keep=math.nan)), (ARG, dict(keep=math.inf)), (ARG, dict(scratch=None)), (WORKSPACE, dict(scratch=X + 8)),
           (WORKSPACE, dict(nbytes=100)), (ARG, dict(scores=_slots(data=None))), (ARG, dict(scores=_slots(data=X + 2))), (ARG, dict(scores=_slots(token=0))), (ARG, dict(scores=_slots(head=0))),
           (ARG, dict(scores=_slots(page=31))), (ARG, dict(scores=_slots(page=-1))), (ARG, dict(scores=_slots(head=BIG + 1))), (BADCFG, dict(q=_heads(n=3))), (BADCFG, dict(q=_heads(n=130))),
           (ARG, dict(anc=X, window=5)), (ARG, dict(anc=X + 4)), (ARG, dict(q=_heads(data=X + 1))), (BADCFG, dict(cache=_cache(dtype=2))), (ARG, dict(batch=_batch(batch=2 ** 30 + 1))),
           (ARG, dict(batch=_batch(max_new=129), anc=X))]
    for code, change in bad:
        assert _weights(lib, **change) == code, change
    assert _weights(lib, tokens=0) == 0 and _weights(lib, tokens=0, lse=None) == 0
    n = ctypes.c_size_t()
    for args in ((-1, 4, 128), (4, 0, 128)):
        assert lib.esp_paged_key_weights_scratch_bytes(*args, ctypes.byref(n)) == ARG
    assert lib.esp_paged_key_weights_scratch_bytes(4, 4, 96, ctypes.byref(n)) == BADCFG and lib.esp_paged_key_weights_scratch_bytes(4, 4, 64, None) == ARG


def _evict(lib, cache=None, batch=None, scores=None, positions=None, seen=None, settled=None, recent=0, budget=X, out=2 * X, scratch=X, nbytes=1 << 30):  # noqa: F811
    return lib.esp_paged_evict(_ref(cache or _cache()), _ref(batch or _batch()), _ref(scores or _slots()), _ref(positions), seen, settled, recent, budget, out, scratch, nbytes, None)


def test_evict_refusals(lib):  # noqa: F811
    bad = [(ARG, dict(recent=-1)), (ARG, dict(positions=_slots())), (ARG, dict(positions=_slots(), seen=X)), (ARG, dict(seen=X, settled=X)), (ARG, dict(budget=None)), (ARG, dict(budget=X + 2)),
           (ARG, dict(out=None)), (ARG, dict(out=X + 1)), (WORKSPACE, dict(scratch=None)), (WORKSPACE, dict(scratch=X + 16)), (WORKSPACE, dict(nbytes=8)), (ARG, dict(scores=_slots(page=20))),
           (ARG, dict(positions=_slots(page=20), seen=X, settled=X)), (ARG, dict(positions=_slots(), seen=X + 2, settled=X)), (BADCFG, dict(cache=_cache(dtype=3)))]
    for code, change in bad:
        assert _evict(lib, **change) == code, change
    assert _evict(lib, batch=_batch(batch=0), budget=None, out=None, scratch=None) == 0
    # slots that are written must not share elements
    assert _evict(lib, cache=_cache(token_stride=64)) == ARG
    n = ctypes.c_size_t()
    for args in ((-1, 2, 100), (2, 0, 100), (2, 2, -1), (2 ** 30 + 1, 2, 100), (2, 2, 2 ** 30 + 1), (2 ** 30, 2 ** 20, 2 ** 30)):
        assert lib.esp_paged_evict_scratch_bytes(*args, ctypes.byref(n)) == ARG, args
    assert lib.esp_paged_evict_scratch_bytes(3, 2, 101, ctypes.byref(n)) == 0 and n.value >= 3 * 2 * 51 * 8


def _accept(lib, tokens=4, cache=None, batch=None, parents=X, drafted=X, chosen=X, out=X, rows=None, stride=4, n_out=X, kv_out=7 * X):  # noqa: F811
    return lib.esp_paged_accept(tokens, _ref(cache or _cache()), _ref(batch or _batch()), parents, drafted, chosen, out, rows, stride, n_out, kv_out, None)


def test_accept_refusals(lib):  # noqa: F811
    b = _batch()
    bad = [(ARG, dict(tokens=-1)), (ARG, dict(parents=None)), (ARG, dict(drafted=None)), (ARG, dict(chosen=None)), (ARG, dict(out=None)), (ARG, dict(n_out=None)), (ARG, dict(kv_out=None)),
           (ARG, dict(parents=X + 1)), (ARG, dict(rows=X + 2)), (ARG, dict(stride=b.max_new - 1)), (ARG, dict(batch=_batch(max_new=129), stride=200)), (ARG, dict(kv_out=b.kv_len)),
           (ARG, dict(kv_out=b.kv_len + 4 * (b.batch - 1))), (BADCFG, dict(cache=_cache(dtype=2))), (ARG, dict(cache=_cache(token_stride=64)))]
    for code, change in bad:
        assert _accept(lib, **change) == code, change
    assert _accept(lib, batch=_batch(batch=0), out=None, n_out=None, kv_out=None) == 0


def _sample(lib, dtype=0, rows=2, vocab=100, logits=X, stride=100, sampling=True, t=None, k=None, p=None, m=None, u=X, tokens=X, logprob=None, scratch=X, nbytes=1 << 40):  # noqa: F811
    s = P.esp_sampling(t, k, p, m) if sampling else None
    return lib.esp_sample(dtype, rows, vocab, logits, stride, _ref(s), u, tokens, logprob, scratch, nbytes, None)


def test_sample_refusals(lib):  # noqa: F811
    bad = [(BADCFG, dict(dtype=2)), (ARG, dict(rows=-1)), (ARG, dict(rows=2 ** 24 + 1)), (ARG, dict(vocab=0)), (ARG, dict(vocab=2 ** 21 + 1)), (ARG, dict(logits=None)), (ARG, dict(logits=X + 2)),
           (ARG, dict(dtype=1, logits=X + 1)), (ARG, dict(stride=-1)), (ARG, dict(stride=BIG + 1)), (ARG, dict(sampling=False)), (ARG, dict(t=X + 2)), (ARG, dict(k=X + 1)), (ARG, dict(p=X + 2)),
           (ARG, dict(m=X + 2)), (ARG, dict(u=None)), (ARG, dict(u=X + 2)), (ARG, dict(tokens=None)), (ARG, dict(tokens=X + 2)), (ARG, dict(logprob=X + 2)), (WORKSPACE, dict(scratch=None)),
           (WORKSPACE, dict(scratch=X + 4)), (WORKSPACE, dict(nbytes=100)), (ARG, dict(rows=2 ** 24, vocab=2 ** 21, nbytes=1 << 62))]
    for code, change in bad:
        assert _sample(lib, **change) == code, change
    assert _sample(lib, rows=0, logits=None, u=None, tokens=None, scratch=None) == 0
    n = ctypes.c_size_t()
    for args in ((-1, 100), (1, 0), (1, 2 ** 21 + 1), (2 ** 24 + 1, 10)):
        assert lib.esp_sample_scratch_bytes(*args, ctypes.byref(n)) == ARG


def test_what_the_binding_refuses():
    """Tensors that do not fit together are refused before the library is called."""
    f, i = (lambda *s: torch.zeros(*s)), (lambda *s: torch.zeros(*s, dtype=torch.int32))
    for bad in (lambda: P.PagedSlots(f(2, 3)), lambda: P.PagedSlots(f(2, 3, 4).double()), lambda: P.PagedSlots(f(2, 3, 4), order="page")):
        with pytest.raises(P.EspError):
            bad()
    k = f(5, 2, 16, 64)
    cache = P.PagedCache(k, k.clone())
    batch = P.PagedBatch(i(3), i(2), i(2, 4), 1)
    slots = P.PagedSlots(f(5, 2, 16))
    from paper_2603_17942_b200 import binding as B
    assert B._slots(slots, cache, torch.float32, "x", "scores") is slots.ref
    for wrong in (P.PagedSlots(f(5, 16, 2)), P.PagedSlots(f(4, 2, 16)), P.PagedSlots(i(5, 2, 16))):
        with pytest.raises(P.EspError):
            B._slots(wrong, cache, torch.float32, "x", "scores")
    assert B._slots(P.PagedSlots(f(5, 16, 2), order="token"), cache, torch.float32, "x", "scores") is not None
    # tensors of no GPU
    for call in (lambda: P.esp_paged_key_weights(cache, batch, f(2, 4, 64), f(2, 4), slots, f(4), 16), lambda: P.esp_paged_evict(cache, batch, slots, i(2), i(2), f(4), 16),
                 lambda: P.esp_paged_accept(cache, batch, i(2), i(2), i(2), i(2, 1), i(2), i(2)), lambda: P.esp_sample(f(2, 100), f(2), i(2), f(4), 16)):
        with pytest.raises(P.EspError):
            call()


def test_scratch_sizes_that_the_binding_refuses():
    from paper_2603_17942_b200 import binding
    scratch = torch.empty(1024, dtype=torch.uint8)
    assert binding._scratch(scratch, 1024, -1, "here") == scratch.data_ptr()
    for size in (-1, 1025, 2 ** 63):
        with pytest.raises(P.EspError):
            binding._scratch(scratch, size, -1, "here")
    with pytest.raises(P.EspError):
        binding._scratch(scratch[::2], 100, -1, "here")
