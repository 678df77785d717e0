"""What the binding and the C entry points of the operators over a paged cache hand over and refuse (no GPU: nothing is launched)."""
import ctypes
import types

import pytest
import torch

import paper_2603_17942_b200 as P
from paper_2603_17942_b200 import binding
from tests.test_paged_host import ARG, X, _batch, _cache, _heads, _norm_rope, lib  # noqa: F401


def test_a_call_without_a_stream_runs_on_the_current_one(monkeypatch):
    """Tensors are used on torch's current stream: a call without one of its own is ordered with them."""
    stream = types.SimpleNamespace(cuda_stream=0x1234)
    monkeypatch.setattr(binding, "_torch", types.SimpleNamespace(cuda=types.SimpleNamespace(current_stream=lambda: stream)))
    assert binding._stream(None) == 0x1234
    assert binding._stream(types.SimpleNamespace(cuda_stream=0x99)) == 0x99 and binding._stream(0) == 0


def test_the_status_of_another_device_is_not_read():
    """The stream that is waited for is the current device's: a batch that is elsewhere is refused as in the other calls."""
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    batch = P.PagedBatch(i(3), i(2), i(2, 4), 1, i(1))
    with pytest.raises(P.EspError) as e:
        P.esp_paged_status(batch)
    assert e.value.code == -8


def test_rows_that_share_elements_are_refused_at_every_size(lib):  # noqa: F811
    """Heads or tokens whose span is 2^64 elements: it does not wrap around to nothing."""
    # token 2^20 of a head stands where token 0 of the next head does
    far = dict(n=2 ** 24 + 1, tok=2 ** 20, head=2 ** 40)
    assert _norm_rope(lib, q=_heads(**far), q_out=_heads(data=2 * X, **far), tokens=2 ** 20 + 1) == ARG
    # head 2^19 of a token stands where head 0 of the next token does
    far = dict(n=2 ** 20, tok=2 ** 40, head=2 ** 21)
    assert _norm_rope(lib, q=_heads(**far), q_out=_heads(data=2 * X, **far), tokens=2 ** 24 + 1) == ARG
    # more heads than a call takes (their sum over queries, keys and values is counted in 32 bits)
    many = dict(n=2 ** 20 + 1, tok=(2 ** 20 + 1) * 128, head=128)
    assert _norm_rope(lib, q=_heads(**many), q_out=_heads(data=2 * X, **many)) == ARG


def _append(lib, cache=None, batch=None, k=None, v=None, q=None, q_gain=None, k_gain=None, positions=None, q_out=None, tokens=4):  # noqa: F811
    r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return lib.esp_paged_append(tokens, r(cache or _cache()), r(batch or _batch()), r(k or _heads()), r(v or _heads(data=3 * X)), r(q), q_gain, k_gain, 1e-6, None, None, positions,
                                r(q_out), None)


def _attend(lib, cache=None, batch=None, anc=None, lse=None, tokens=4):  # noqa: F811
    r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return lib.esp_paged_attention(tokens, r(cache or _cache()), r(batch or _batch()), r(_heads(n=4)), anc, 0, 0.0, r(_heads(n=4, data=4 * X)), lse, X,
                                   P.esp_paged_attention_scratch_bytes(4, 128), None)


def test_more_sequences_than_the_kernels_count(lib):  # noqa: F811
    """The kernels deal 32 lanes their shares of the sequences in 32 bits: above 2^30 of them nothing would be walked, and nobody told."""
    batch = _batch(batch=2 ** 30 + 1)
    assert _append(lib, batch=batch) == ARG and _attend(lib, batch=batch) == ARG
    assert _append(lib, batch=_batch(batch=2 ** 30), tokens=0) == 0 and _attend(lib, batch=_batch(batch=2 ** 30), tokens=0) == 0


def test_addresses_off_their_types_alignment(lib):  # noqa: F811
    """A kernel that reads a gain, a length or a mask off its type's alignment would fault: the host says so first."""
    q, o = _heads(), _heads(data=2 * X)
    for gain in ("q_gain", "k_gain"):
        both = dict(q=q, q_out=o, k=_heads(data=3 * X), k_out=_heads(data=4 * X))
        assert _norm_rope(lib, **both, **{gain: X + 1}) == ARG and _norm_rope(lib, **both, dtype=0, **{gain: X + 2}) == ARG
        assert _append(lib, q=_heads(n=4), q_out=_heads(n=4, data=4 * X), **{gain: X + 1}) == ARG
        assert _norm_rope(lib, **both, **{gain: X + 2}, tokens=0) == 0
    assert _norm_rope(lib, q=q, q_out=o, positions=X + 2) == ARG and _append(lib, positions=X + 1) == ARG
    for name in ("q_start", "kv_len", "page_table", "status"):
        batch = _batch(**{name: X + 2})
        assert _append(lib, batch=batch) == ARG and _attend(lib, batch=batch) == ARG, name
    assert _attend(lib, anc=X + 4) == ARG and _attend(lib, lse=X + 2) == ARG
    assert _attend(lib, anc=X + 8, lse=X + 4, tokens=0) == 0
    assert lib.esp_paged_status(X + 1, None, None) == ARG


def test_append_into_slots_that_share_elements(lib):  # noqa: F811
    """Every stride spans a head, but two tokens' slots are one: nothing is written there.  Slots in any order of nesting are fine, and so is reading them."""
    for strides in (dict(head_stride=1024), dict(page_stride=2048), dict(page_stride=128, token_stride=256, head_stride=4096), dict(page_stride=2 ** 40, token_stride=128, head_stride=2 ** 40),
                    dict(token_stride=192, head_stride=256)):
        assert _append(lib, cache=_cache(**strides)) == ARG, strides
        assert _append(lib, cache=_cache(**strides), tokens=0) == ARG and _attend(lib, cache=_cache(**strides), tokens=0) == 0
    for strides in (dict(), dict(page_stride=128, token_stride=1024, head_stride=16384), dict(token_stride=256, head_stride=128), dict(page_stride=128, token_stride=2048, head_stride=1024)):
        assert _append(lib, cache=_cache(**strides), tokens=0) == 0, strides
    assert _append(lib, cache=_cache(page_size=1, token_stride=0, head_stride=128, page_stride=256), tokens=0) == 0


def test_numbers_that_do_not_fit_are_not_cut_off(lib):  # noqa: F811
    """2^32 + 5 is not 5: numbers that the library takes in 32 bits are checked before they are handed over."""
    far = 2 ** 32
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    k = torch.zeros(4, 2, 16, 64)
    cache, batch, x = P.PagedCache(k, k.clone()), P.PagedBatch(i(3), i(2), i(2, 4), 1), torch.zeros(2, 2, 64)
    many = torch.zeros(1, 1, 64).expand(far + 2, 2, 64)
    calls = {
        "max_new": lambda: P.PagedBatch(i(3), i(2), i(2, 4), far + 1),
        "page_table": lambda: P.PagedBatch(i(3).to("meta"), i(2).to("meta"), torch.empty(2, far, dtype=torch.int32, device="meta")[:, :4], 1),
        "rotary_dim": lambda: P.rope_cfg(far + 64),
        "original_len": lambda: P.rope_cfg(64, scaling="linear", factor=2.0, original_len=far + 8192),
        "n_q_heads": lambda: P.esp_paged_attention_scratch_bytes(far + 4, 64),
        "head_dim": lambda: P.esp_paged_attention_scratch_bytes(4, far + 64),
        "window": lambda: P.esp_paged_attention(cache, batch, x, x.clone(), torch.zeros(8), 32, window=far + 5),
        "tokens": lambda: P.esp_paged_attention(cache, batch, many, many, torch.zeros(8), 32),
        "tokens ": lambda: P.esp_paged_append(cache, batch, many, many),
        "tokens  ": lambda: P.esp_qk_norm_rope(many, None, many, None),
    }
    for what, call in calls.items():
        with pytest.raises(P.EspError, match=what.strip()):
            call()
    with pytest.raises(P.EspError):
        P.PagedCache(k[:1].expand(far + 1, 2, 16, 64), k[:1].expand(far + 1, 2, 16, 64))
    assert P.PagedBatch(i(3), i(2), i(2, 4), 2 ** 31 - 1).c.max_new == 2 ** 31 - 1
