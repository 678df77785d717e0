"""The operators over a paged cache as far as they go without a GPU: frequencies of the rotation, the structs of the binding, refusals."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2603_17942_b200 as P
from paper_2603_17942_b200 import build as esp_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARG, BADCFG, WORKSPACE = -8, -1, -2


@pytest.fixture(scope="module")
def lib():
    esp_build.build()
    return P.load_library()


def test_structs_mirror_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "esp.h")).read(), flags=re.S)
    for cname, ctype in (("esp_heads", P.esp_heads), ("esp_paged_cache", P.esp_paged_cache), ("esp_paged_batch", P.esp_paged_batch), ("esp_rope_cfg", P.esp_rope_cfg)):
        end = text.index("} %s;" % cname)
        body = text[text.rindex("typedef struct {", 0, end) + len("typedef struct {"):end]
        members = [n.strip().lstrip("*").strip() for d in body.split(";") if d.strip()
                   for n in re.sub(r"^(const\s+)?\w+\s*\*?", "", d.strip(), count=1).split(",")]
        assert members == [f[0] for f in ctype._fields_], cname
    assert re.search(r"#define\s+ESP_ROPE_MAX_DIM\s+%d" % P.ESP_ROPE_MAX_DIM, text)


# ---------------------------------------------------------------- frequencies
def _plain(r, base):
    return base ** (-2.0 * np.arange(r // 2) / r)


def test_frequencies_of_every_scaling(lib):
    """The formulas of the header in fp64 (relative error of a few 2^-53; 1e-13 covers powers and logarithms)."""
    for r, base, factor, orig in ((128, 10000.0, 4.0, 4096), (64, 500000.0, 8.0, 8192), (20, 10000.0, 2.0, 2048), (4, 100.0, 32.0, 100)):
        f = _plain(r, base)
        got = P.esp_rope_frequencies(P.rope_cfg(r, base))
        assert np.allclose(got, f, rtol=1e-13, atol=0)
        assert np.allclose(P.esp_rope_frequencies(P.rope_cfg(r, base, scaling="linear", factor=factor)), f / factor, rtol=1e-13, atol=0)
        grown = base * factor ** (r / (r - 2))
        assert np.allclose(P.esp_rope_frequencies(P.rope_cfg(r, base, scaling="base", factor=factor)), _plain(r, grown), rtol=1e-13, atol=0)
        got = P.esp_rope_frequencies(P.rope_cfg(r, base, scaling="rotations", factor=factor, original_len=orig, low=1.0, high=4.0))
        for i in range(r // 2):
            turns = orig * f[i] / (2 * math.pi)
            w = (turns - 1) / 3
            want = f[i] / factor if turns < 1 else f[i] if turns > 4 else f[i] * (w + (1 - w) / factor)
            assert abs(got[i] - want) <= 1e-13 * want
        got = P.esp_rope_frequencies(P.rope_cfg(r, base, scaling="index", factor=factor, original_len=orig, low=1.0, high=32.0))
        first = max(math.floor(r * math.log(orig / (32 * 2 * math.pi)) / (2 * math.log(base))), 0)
        last = min(math.ceil(r * math.log(orig / (2 * math.pi)) / (2 * math.log(base))), r - 1)
        for i in range(r // 2):
            w = 1 - min(max((i - first) / max(last - first, 0.001), 0), 1)
            assert abs(got[i] - f[i] * (w + (1 - w) / factor)) <= 1e-13 * f[i]


def test_frequencies_against_a_library_of_models(lib):
    """The forms that published checkpoints name, computed in fp32 there: 1e-6 relative is a few of its roundings."""
    utils = pytest.importorskip("transformers.modeling_rope_utils")
    config = pytest.importorskip("transformers").LlamaConfig
    make = lambda **rope: config(hidden_size=4096, num_attention_heads=32, head_dim=128, max_position_embeddings=32768, rope_parameters=rope)  # noqa: E731
    try:
        cfgs = {"linear": make(rope_type="linear", factor=4.0, rope_theta=10000.0),
                "llama3": make(rope_type="llama3", factor=8.0, low_freq_factor=1.0, high_freq_factor=4.0, original_max_position_embeddings=8192, rope_theta=500000.0),
                "yarn": make(rope_type="yarn", factor=4.0, original_max_position_embeddings=8192, beta_fast=32.0, beta_slow=1.0, rope_theta=1000000.0)}
        found = {k: utils.ROPE_INIT_FUNCTIONS[k](c, torch.device("cpu")) for k, c in cfgs.items()}
    except (TypeError, KeyError, AttributeError) as e:
        pytest.skip(f"another interface: {e}")
    ours = {"linear": P.rope_cfg(128, 10000.0, scaling="linear", factor=4.0),
            "llama3": P.rope_cfg(128, 500000.0, scaling="rotations", factor=8.0, original_len=8192),
            "yarn": P.rope_cfg(128, 1000000.0, scaling="index", factor=4.0, original_len=8192)}
    for name, (inv_freq, _) in found.items():
        got = P.esp_rope_frequencies(ours[name])
        assert np.allclose(got, inv_freq.double().numpy(), rtol=2e-6, atol=0), name


@pytest.mark.parametrize("change", [dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=258), dict(scaling=5), dict(scaling=-1), dict(interleaved=2), dict(base=0.0),
                                    dict(base=-2.0), dict(base=math.nan), dict(base=math.inf), dict(amplitude=math.nan), dict(scaling=1, factor=0.0),
                                    dict(scaling=1, factor=math.inf), dict(scaling=2, rotary_dim=2), dict(scaling=3, original_len=0), dict(scaling=3, low=4.0),
                                    dict(scaling=4, low=0.0), dict(scaling=4, high=math.inf), dict(scaling=4, base=1.0)])
def test_rope_configurations_that_are_refused(lib, change):
    cfg = P.rope_cfg(64, 10000.0, factor=2.0, original_len=4096)
    cfg.high = 4.0
    for k, v in change.items():
        setattr(cfg, k, v)
    for call in (lambda: P.esp_rope_frequencies(cfg), lambda: P.esp_rope_table_bytes(cfg)):
        with pytest.raises(P.EspError) as e:
            call()
        assert e.value.code == BADCFG
    with pytest.raises(P.EspError):
        P.rope_cfg(64, scaling="other")


# ---------------------------------------------------------------- refusals of the C entry points (nothing is launched: the pointers are never followed)
X = 0x100000       # an address that is aligned for everything


def _heads(n=2, tok=1024, head=128, data=X):
    return P.esp_heads(data, tok, head, n)


def _norm_rope(lib, dtype=1, tokens=4, dim=128, q=None, k=None, q_gain=None, k_gain=None, eps=1e-6, rope=None, table=None, positions=X, q_out=None, k_out=None):
    r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return lib.esp_qk_norm_rope(dtype, tokens, dim, r(q), r(k), q_gain, k_gain, eps, r(rope), table, positions, r(q_out), r(k_out), None)


def test_norm_rope_refusals(lib):
    q, o = _heads(), _heads(data=2 * X)
    rope = P.rope_cfg(128)
    bad = [
        (ARG, dict()), (ARG, dict(q=q)), (ARG, dict(q_out=o)), (ARG, dict(q=q, k_out=o)), (ARG, dict(q=q, q_out=o, tokens=-1)), (ARG, dict(q=q, q_out=o, tokens=2 ** 30 + 1)),
        (BADCFG, dict(q=q, q_out=o, dtype=2)), (BADCFG, dict(q=q, q_out=o, dim=0)), (BADCFG, dict(q=q, q_out=o, dim=257)),
        (ARG, dict(q=q, q_out=_heads(n=3, data=2 * X))), (ARG, dict(q=q, q_out=o, k_gain=X)), (ARG, dict(q=q, q_out=o, eps=-1.0)), (ARG, dict(q=q, q_out=o, eps=math.nan)),
        (ARG, dict(q=q, q_out=o, rope=rope, table=X, positions=None)), (ARG, dict(q=q, q_out=o, rope=rope)), (ARG, dict(q=q, q_out=o, rope=rope, table=X + 8)),
        (BADCFG, dict(q=q, q_out=o, rope=rope, table=X, dim=64)),
        (ARG, dict(q=_heads(data=None), q_out=o)), (ARG, dict(q=_heads(data=X + 1), q_out=o)), (ARG, dict(q=_heads(data=X + 2), q_out=o, dtype=0)),
        (ARG, dict(q=_heads(tok=-1), q_out=o)), (ARG, dict(q=_heads(n=0), q_out=_heads(n=0, data=2 * X))),
        (ARG, dict(q=q, q_out=_heads(tok=0, data=2 * X))), (ARG, dict(q=q, q_out=_heads(head=64, data=2 * X))), (ARG, dict(q=q, q_out=_heads(tok=192, data=2 * X))),
        (ARG, dict(q=q, q_out=_heads(tok=2048))),
    ]
    for code, kw in bad:
        assert _norm_rope(lib, **kw) == code, kw
    assert _norm_rope(lib, q=q, q_out=o, tokens=0) == 0


def _cache(**kw):
    c = dict(k=X, v=2 * X, page_stride=4096, token_stride=128, head_stride=2048, n_pages=8, page_size=16, n_kv_heads=2, head_dim=128, dtype=1)
    c.update(kw)
    return P.esp_paged_cache(*c.values())


def _batch(**kw):
    c = dict(batch=2, max_new=4, q_start=X, kv_len=X, page_table=X, table_pages=4, table_stride=4, status=None)
    c.update(kw)
    return P.esp_paged_batch(*c.values())


BAD_CACHES = [(ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(n_pages=0)), (ARG, dict(page_size=0)), (ARG, dict(n_kv_heads=0)), (BADCFG, dict(dtype=2)),
              (BADCFG, dict(head_dim=96)), (ARG, dict(k=X + 1)), (ARG, dict(page_stride=-4096)), (ARG, dict(token_stride=64)), (ARG, dict(head_stride=0)), (ARG, dict(page_stride=0))]
BAD_BATCHES = [(ARG, dict(batch=-1)), (ARG, dict(max_new=-1)), (ARG, dict(q_start=None)), (ARG, dict(kv_len=None)), (ARG, dict(page_table=None)), (ARG, dict(table_pages=0)),
               (ARG, dict(table_stride=3))]


def test_append_refusals(lib):
    def call(cache={}, batch={}, k=_heads(), v=_heads(data=3 * X), q=None, q_gain=None, eps=1e-6, rope=None, table=None, q_out=None, tokens=4):
        r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
        return lib.esp_paged_append(tokens, r(_cache(**cache)), r(_batch(**batch)), r(k), r(v), r(q), q_gain, None, eps, r(rope), table, None, r(q_out), None)
    for code, kw in BAD_CACHES:
        assert call(cache=kw) == code, kw
    for code, kw in BAD_BATCHES:
        assert call(batch=kw) == code, kw
    q, o = _heads(n=4), _heads(n=4, data=4 * X)
    for code, kw in [(ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(k=_heads(n=3))), (ARG, dict(v=_heads(n=1))), (ARG, dict(q=q)), (ARG, dict(q_out=o)),
                     (ARG, dict(q=q, q_out=_heads(n=2, data=4 * X))), (ARG, dict(q_gain=X)), (ARG, dict(tokens=-1)), (ARG, dict(tokens=2 ** 30 + 1)), (ARG, dict(eps=math.nan)), (ARG, dict(rope=P.rope_cfg(128))),
                     (BADCFG, dict(rope=P.rope_cfg(256), table=X)), (ARG, dict(q=q, q_out=_heads(n=4, tok=300, data=4 * X)))]:
        assert call(**kw) == code, kw
    assert call(tokens=0) == 0 and call(batch=dict(batch=0)) == 0 and call(batch=dict(max_new=0)) == 0


def test_attention_refusals(lib):
    need = P.esp_paged_attention_scratch_bytes(4, 128)

    def call(cache={}, batch={}, q=_heads(n=4), out=_heads(n=4, data=4 * X), anc=None, window=0, scale=0.0, scratch=X, nbytes=need, tokens=4):
        r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
        return lib.esp_paged_attention(tokens, r(_cache(**cache)), r(_batch(**batch)), r(q), anc, window, scale, r(out), None, scratch, nbytes, None)
    for code, kw in BAD_CACHES:
        assert call(cache=kw) == code, kw
    for code, kw in BAD_BATCHES:
        assert call(batch=kw) == code, kw
    for code, kw in [(ARG, dict(q=None)), (ARG, dict(out=None)), (ARG, dict(scratch=None)), (WORKSPACE, dict(nbytes=need - 1)), (WORKSPACE, dict(scratch=X + 16)),
                     (ARG, dict(window=-1)), (ARG, dict(scale=-1.0)), (ARG, dict(scale=math.nan)), (ARG, dict(scale=math.inf)), (ARG, dict(tokens=-1)), (ARG, dict(tokens=2 ** 30 + 1)),
                     (ARG, dict(out=_heads(n=4))), (ARG, dict(out=_heads(n=2, data=4 * X))), (BADCFG, dict(q=_heads(n=5), out=_heads(n=5, data=4 * X))),
                     (BADCFG, dict(q=_heads(n=130), out=_heads(n=130, tok=130 * 128, data=4 * X))),
                     (ARG, dict(anc=X, window=5)), (ARG, dict(anc=X, batch=dict(max_new=129))), (ARG, dict(out=_heads(n=4, tok=64, data=4 * X)))]:
        assert call(**kw) == code, kw
    assert call(tokens=0) == 0 and call(batch=dict(batch=0)) == 0 and call(batch=dict(max_new=0)) == 0
    for bad in ((0, 128), (4, 96)):
        with pytest.raises(P.EspError):
            P.esp_paged_attention_scratch_bytes(*bad)


def test_the_binding_takes_no_tensors_of_the_host():
    k = torch.zeros(4, 2, 16, 64)
    with pytest.raises(P.EspError):
        P.PagedCache(k, k, order="other")
    with pytest.raises(P.EspError):
        P.PagedCache(k, k.bfloat16())
    with pytest.raises(P.EspError):
        P.PagedCache(k.half(), k.half())
    with pytest.raises(P.EspError):
        P.PagedCache(k.transpose(2, 3), k.transpose(2, 3))
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    for args in ((i(3), i(3), i(3, 4)), (i(4), i(3), i(2, 4)), (i(4).long(), i(3), i(3, 4)), (i(4), i(3), i(3, 4).long()), (i(4), i(3), i(4, 3).t())):
        with pytest.raises(P.EspError):
            P.PagedBatch(*args, 1)
    cache, batch = P.PagedCache(k, k.clone()), P.PagedBatch(i(3), i(2), i(2, 4), 1)
    x = torch.zeros(2, 2, 64)
    for call in (lambda: P.esp_paged_append(cache, batch, x, x), lambda: P.esp_paged_attention(cache, batch, x, x.clone(), torch.zeros(8), 32),
                 lambda: P.esp_qk_norm_rope(x, None, x, None)):
        with pytest.raises(P.EspError) as e:
            call()
        assert e.value.code == ARG
