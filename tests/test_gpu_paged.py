"""The operators over a paged cache on the GPU, against plain implementations in 64 bits.

Roundings: to bf16 at most 2^-8 of the value, to fp32 2^-24.  Every tolerance is counted from them where it stands.
"""
import math

import numpy as np
import pytest
import torch

import paper_2603_17942_b200 as P

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}       # one rounding, relative
NAN = float("nan")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


# ================================================================ norm and rotation
def _rope_table(cfg):
    t = torch.empty(P.esp_rope_table_bytes(cfg), dtype=torch.uint8, device="cuda")
    P.esp_rope_table(cfg, t)
    return t


def _norm_rope_ref(x, positions, cfg, gain, eps):
    """In 64 bits, angles in the host's extended precision; (result, length of the pair that each element belongs to)."""
    y = x.double().cpu().numpy()
    if gain is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * gain.double().cpu().numpy()
    out, length = y.copy(), np.abs(y)
    if cfg is not None:
        r = cfg.rotary_dim
        angle = np.asarray(positions, np.int64).astype(np.longdouble)[:, None] * P.esp_rope_frequencies(cfg).astype(np.longdouble)
        c, s = (np.float64(cfg.amplitude) * f(angle).astype(np.float64) for f in (np.cos, np.sin))
        i = np.arange(r // 2)
        ia, ib = (2 * i, 2 * i + 1) if cfg.interleaved else (i, i + r // 2)
        a, b = y[..., ia], y[..., ib]
        out[..., ia], out[..., ib] = a * c[:, None] - b * s[:, None], b * c[:, None] + a * s[:, None]
        length[..., ia] = length[..., ib] = np.hypot(a, b) * abs(cfg.amplitude)
    return out, length


def _check_norm_rope(got, x, positions, cfg, gain, eps, dtype):
    """fp32 arithmetic: the norm's sum and root 14 roundings, angle, sine, amplitude, products and sum 10 of the pair's length: 32 * 2^-24 of it; a frequency
    rounded to fp64 turns a position of 2^31 by another 2^-22 / 2 in this reference: 2^-23 * |p| / 2^31 of the length."""
    ref, length = _norm_rope_ref(x, positions, cfg, gain, eps)
    far = np.abs(np.asarray(positions, np.float64))[:, None, None] * 2.0 ** -52 if cfg is not None else 0.0
    tol = HALF[dtype] * np.abs(ref) * 1.0001 + (32 * 2.0 ** -24 + far) * length + 1e-30
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= tol).all(), f"worst {np.max(err / tol)} of the tolerance"


ROPES = [None, dict(share=1.0), dict(share=1.0, interleaved=True), dict(share=0.5, scaling="linear", factor=4.0),
         dict(share=0.25, interleaved=True, scaling="index", factor=8.0, amplitude=1.2), dict(share=-1, scaling="rotations", factor=8.0)]


def _cfg(spec, D):
    if spec is None:
        return None
    kw = {k: v for k, v in spec.items() if k != "share"}
    r = max(2, int(D * spec["share"]) // 2 * 2) if spec["share"] > 0 else max(2, (D * 3 // 4) // 2 * 2 - 2)      # the last one: a share that is no power of two
    return P.rope_cfg(r, 10000.0, **kw)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D", [128, 64, 32, 256, 80, 6])
@pytest.mark.parametrize("rope", range(len(ROPES)))
@pytest.mark.parametrize("norm", [False, True])
def test_norm_rope(dtype, D, rope, norm):
    """Head sizes, layouts, shares and scalings, queries and keys with gains of their own, views into one projection output."""
    cfg = _cfg(ROPES[rope], D)
    g = _gen(D * 100 + rope * 10 + norm)
    T, Hq, Hk = 37, 5, 2
    qkv = _randn(g, T, Hq + Hk + 1, D, dtype=DT[dtype])
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    gains = [(1 + 0.2 * _randn(g, D)).to(DT[dtype]) if norm else None for _ in range(2)]
    pos = torch.randint(0, 5000, (T,), generator=g, device="cuda", dtype=torch.int32)
    q_out, k_out = torch.full((T, Hq, D), NAN, device="cuda", dtype=DT[dtype]), torch.full((Hk, T, D), NAN, device="cuda", dtype=DT[dtype]).transpose(0, 1)
    P.esp_qk_norm_rope(q, k, q_out, k_out, cfg, None if cfg is None else _rope_table(cfg), pos, gains[0], gains[1], eps=1e-5)
    p = pos.cpu().numpy()
    _check_norm_rope(q_out, q, p, cfg, gains[0], 1e-5, dtype)
    _check_norm_rope(k_out, k, p, cfg, gains[1], 1e-5, dtype)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D", [("fp32", 64), ("bf16", 128), ("fp32", 34)])
def test_rotation_of_far_and_negative_positions(dtype, D, interleaved):
    cfg = P.rope_cfg(D, 500000.0, interleaved=interleaved)
    pos = torch.tensor([0, 1, -1, 131071, 1 << 20, (1 << 24) + 1, -(1 << 24) - 3, 10 ** 9 + 7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    x = _randn(_gen(3), len(pos), 3, D, dtype=DT[dtype])
    out = torch.empty_like(x)
    P.esp_qk_norm_rope(x, None, out, None, cfg, _rope_table(cfg), pos)
    _check_norm_rope(out, x, pos.cpu().numpy(), cfg, None, 0, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,H,D", [(1, 1, 64), (1, 40, 128), (3, 1, 32), (300, 12, 128), (2000, 3, 64)])
def test_norm_rope_in_place_equals_out_of_place(dtype, T, H, D):
    cfg = P.rope_cfg(D // 2, 10000.0)
    g = _gen(T)
    x = _randn(g, T, H, D, dtype=DT[dtype])
    gain = _randn(g, D, dtype=DT[dtype])
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    out, table = torch.empty_like(x), _rope_table(cfg)
    P.esp_qk_norm_rope(None, x, None, out, cfg, table, pos, k_gain=gain)
    _check_norm_rope(out, x, pos.cpu().numpy(), cfg, gain, 1e-6, dtype)
    P.esp_qk_norm_rope(None, x, None, x, cfg, table, pos, k_gain=gain)
    assert torch.equal(out, x)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("what", ["offset", "head stride", "token stride", "broadcast"])
def test_norm_rope_of_strides_without_alignment(dtype, what):
    """Tensors that no wide access fits, and one that is read with stride zero; elements between the rows stay as they are."""
    T, H, D = 19, 3, 64
    g = _gen(5)
    pad = {"offset": (0, 0, 1), "head stride": (0, 1, 0), "token stride": (1, 0, 0), "broadcast": (0, 0, 0)}[what]
    hs = D + pad[1]
    ts = H * hs + pad[0]

    def strided(fill):
        flat = torch.full((T * ts + 8,), fill, dtype=DT[dtype], device="cuda")
        return flat, flat[pad[2]:].as_strided((T, H, D), (ts, hs, 1), flat.storage_offset() + pad[2])
    x = strided(0.0)[1]
    x.copy_(_randn(g, T, H, D))
    if what == "broadcast":
        x = x[:1, :1].expand(T, H, D)
    flat, out = strided(7.0)
    cfg = P.rope_cfg(D, 10000.0)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 100
    P.esp_qk_norm_rope(x, None, out, None, cfg, _rope_table(cfg), pos)
    _check_norm_rope(out, x, pos.cpu().numpy(), cfg, None, 0, dtype)
    out.fill_(7.0)
    assert bool((flat == 7.0).all())


def test_norm_rope_of_infinite_and_tiny_rows():
    """A row of zeros stays zero with eps, an infinite element spoils its own head alone."""
    x = torch.randn(3, 2, 128, device="cuda", dtype=torch.bfloat16)
    x[0, 0] = 0
    x[1, 1, 5] = math.inf
    gain = torch.ones(128, device="cuda", dtype=torch.bfloat16)
    pos, out, cfg = torch.arange(3, dtype=torch.int32, device="cuda"), torch.empty_like(x), P.rope_cfg(128)
    P.esp_qk_norm_rope(x, None, out, None, cfg, _rope_table(cfg), pos, q_gain=gain)
    assert bool((out[0, 0] == 0).all()) and bool(torch.isfinite(out[[0, 0, 1, 2, 2], [0, 1, 0, 0, 1]]).all()) and not bool(torch.isfinite(out[1, 1, 5]))


# ================================================================ a batch over pages
class Batch:
    """n[b] new tokens and kv[b] positions with them; pages of the sequences dealt at random, one page behind the last is nobody's."""

    def __init__(self, n, kv, page, Hkv, D, dtype, order="head", seed=0, front=0, back=0, fill=None, status=True, spare_columns=0):
        g = _gen(seed)
        self.n, self.kv, self.page, self.front = n, kv, page, front
        self.tokens = front + sum(n) + back
        need = [-(-t // page) for t in kv]
        total = sum(need) + 1
        order_ = np.random.default_rng(seed).permutation(total)
        width = max(max(need), 1)
        table = np.full((len(n), width + spare_columns), -5, np.int32)
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = order_[at:at + m]
            at += m
        self.table = table[:, :width]
        self.unused = int(order_[-1])
        shape = (total, Hkv, page, D) if order == "head" else (total, page, Hkv, D)
        make = (lambda: torch.full(shape, fill, device="cuda", dtype=DT[dtype])) if fill is not None else (lambda: _randn(g, *shape, dtype=DT[dtype]))
        self.k, self.v, self.order = make(), make(), order
        self.cache = P.PagedCache(self.k, self.v, order=order)
        q_start = front + np.concatenate([[0], np.cumsum(n)])
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda") if status else None
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
        self.q_start, self.kv_len, self.table_d = i32(q_start), i32(kv), i32(table)[:, :width]
        self.batch = P.PagedBatch(self.q_start, self.kv_len, self.table_d, max(n + [1]), self.status)

    def slots(self, b):
        """(page, slot) of positions 0 .. kv - 1"""
        p = np.arange(self.kv[b])
        return torch.tensor(self.table[b][p // self.page].astype(np.int64), device="cuda"), torch.tensor(p % self.page, device="cuda")

    def view(self, x):
        return x if self.order == "token" else x.transpose(1, 2)          # [page, slot, head, D]

    def read(self, x, b):
        page, slot = self.slots(b)
        return self.view(x)[page, slot]                                   # [kv, Hkv, D]

    def ok(self):
        assert self.status is None or P.esp_paged_status(self.batch) == 0


def _scratch(Hq, D):
    nb = P.esp_paged_attention_scratch_bytes(Hq, D)
    return torch.full((nb,), 255, dtype=torch.uint8, device="cuda"), nb          # NaN everywhere: contents are of no account


@pytest.mark.parametrize("dtype,D,page,order", [("bf16", 128, 16, "head"), ("bf16", 64, 24, "token"), ("fp32", 64, 16, "token"), ("fp32", 32, 7, "head"), ("bf16", 128, 1, "head"),
                                                ("bf16", 32, 256, "token")])
@pytest.mark.parametrize("n,kv", [([1], [1]), ([1], [33]), ([5, 1, 0, 130], [5, 300, 40, 200]), ([3, 4], [1, 9]), ([1] * 70, list(range(1, 71)))])
def test_append(dtype, D, page, order, n, kv):
    """Every slot of the batch gets its key and value, every other element of the pages and of q_out keeps its bits: tokens in front of and behind the
    sequences, positions below zero (kv < n), pages of nobody."""
    Hkv, Hq = 2, 6
    b = Batch(n, kv, page, Hkv, D, dtype, order, seed=sum(kv) + D, front=2, back=3)
    g = _gen(9)
    qkv = _randn(g, b.tokens, Hq + 2 * Hkv, D, dtype=DT[dtype])
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    cfg = P.rope_cfg(D // 2, 10000.0, interleaved=D == 64)
    gain = [(1 + 0.1 * _randn(g, D)).to(DT[dtype]) for _ in range(2)]
    q_out = torch.full((b.tokens, Hq, D), 7.0, device="cuda", dtype=DT[dtype])
    k0, v0 = b.k.clone(), b.v.clone()
    P.esp_paged_append(b.cache, b.batch, k, v, cfg, _rope_table(cfg), k_gain=gain[0], q=q, q_out=q_out, q_gain=gain[1])
    b.ok()
    written = torch.zeros(b.tokens, dtype=torch.bool)
    at = b.front
    for s, (m, t) in enumerate(zip(n, kv)):
        rows = [i for i in range(m) if t - m + i >= 0]
        tok = torch.tensor([at + i for i in rows], dtype=torch.int64)
        pos = np.array([t - m + i for i in rows], np.int64)
        written[tok] = True
        at += m
        if not rows:
            continue
        page_, slot = (x[pos] for x in b.slots(s))
        got_k, got_v = b.view(b.k)[page_, slot], b.view(b.v)[page_, slot]
        assert torch.equal(got_v, v[tok.cuda()])
        _check_norm_rope(got_k, k[tok.cuda()], pos, cfg, gain[0], 1e-6, dtype)
        _check_norm_rope(q_out[tok.cuda()], q[tok.cuda()], pos, cfg, gain[1], 1e-6, dtype)
        b.view(k0)[page_, slot], b.view(v0)[page_, slot] = got_k, got_v
    assert torch.equal(b.k, k0) and torch.equal(b.v, v0)
    assert bool((q_out[~written.cuda()] == 7.0).all())


def test_append_keys_alone_without_rotation_copies_them():
    b = Batch([3, 2], [20, 2], 16, 2, 64, "bf16", seed=4, fill=0.0)
    k, v = (_randn(_gen(s), 5, 2, 64, dtype=torch.bfloat16) for s in (1, 2))
    P.esp_paged_append(b.cache, b.batch, k, v)
    assert torch.equal(b.read(b.k, 0)[17:], k[:3]) and torch.equal(b.read(b.v, 0)[17:], v[:3])
    assert torch.equal(b.read(b.k, 1), k[3:]) and torch.equal(b.read(b.v, 1), v[3:])


def test_append_at_given_positions():
    """The rows of a draft tree share positions: the rotation goes by them, the slots by the rows."""
    n, kv, D = [6], [40], 128
    b = Batch(n, kv, 16, 1, D, "bf16", seed=5)
    depth = np.array([0, 1, 1, 2, 2, 3])
    pos = torch.tensor(34 + depth, dtype=torch.int32, device="cuda")
    k, v = (_randn(_gen(s), 6, 1, D, dtype=torch.bfloat16) for s in (1, 2))
    cfg = P.rope_cfg(D)
    P.esp_paged_append(b.cache, b.batch, k, v, cfg, _rope_table(cfg), positions=pos)
    _check_norm_rope(b.read(b.k, 0)[34:], k, 34 + depth, cfg, None, 0, "bf16")
    assert torch.equal(b.read(b.v, 0)[34:], v)


# ================================================================ attention
def _visible(n, kv, window, anc):
    """[n][kv] truth values"""
    p, j = np.arange(kv - n, kv)[:, None], np.arange(kv)[None]
    if anc is None:
        return (j <= p) & ((j > p - window) if window else True)
    see = np.broadcast_to(j < kv - n, (n, kv)).copy()
    for i in range(n):
        for r in range(n):
            if kv - n + r >= 0:
                see[i, kv - n + r] = bool((int(anc[i][r // 64]) >> (r % 64)) & 1)
    see[(p < 0)[:, 0]] = False
    return see


def _attention(b, q, anc=None, window=0, scale=0.0, lse=True, out=None, stream=None):
    D = q.shape[2]
    out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype) if out is None else out
    ls = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    sc, nb = _scratch(q.shape[1], D)
    P.esp_paged_attention(b.cache, b.batch, q, out, sc, nb, anc=None if anc is None else torch.from_numpy(anc.view(np.int64)).cuda(), window=window, scale=scale, lse=ls,
                          stream=stream)
    return out, ls


def _check_attention(b, q, out, lse, anc=None, window=0, scale=0.0):
    """Against softmax in 64 bits.  A weight is off by the rounding of its bf16 form (none in fp32) and by twice the error of its logit: the sum of D products, the
    scaling and the exponential, (D + 8) 2^-24 of scale |q| |k| and 2^-21; sums over n keys add n 2^-24.  All of it times the sum of weighted |v|, and the output's own
    rounding.  lse: the logit's error, 2^-20 of it and the sum's."""
    dtype = "fp32" if q.dtype == torch.float32 else "bf16"
    D, Hq = q.shape[2], q.shape[1]
    g = Hq // (b.k.shape[1] if b.order == "head" else b.k.shape[2])
    scale = scale or D ** -0.5
    at = b.front
    assert bool((out[:at] == 7.0).all()) and bool((out[at + sum(b.n):] == 7.0).all())
    for s, (n, kv) in enumerate(zip(b.n, b.kv)):
        if n == 0:
            continue
        see = torch.from_numpy(_visible(n, kv, window, None if anc is None else anc[at:at + n])).cuda()
        k, v = b.read(b.k, s).double(), b.read(b.v, s).double()
        x = q[at:at + n].double()
        for h in range(Hq):
            kk, vv = k[:, h // g], v[:, h // g]
            z = (x[:, h] @ kk.T * scale).masked_fill(~see, -math.inf)
            empty = ~see.any(1)
            w = torch.softmax(z.masked_fill(empty[:, None], 0.0), -1) * see
            ref, mag = w @ vv, w @ vv.abs()
            size = scale * x[:, h].norm(dim=1) * kk.norm(dim=1).max()
            logit = (D + 8) * 2.0 ** -24 * size + 2.0 ** -21 + kv * 2.0 ** -24
            p_round = 0.0 if dtype == "fp32" else HALF["bf16"]
            tol = (p_round + 2 * logit)[:, None] * mag * 1.01 + HALF[dtype] * 1.01 * ref.abs() + 1e-30
            got = out[at:at + n, h].double()
            err = (got - ref).abs()
            assert bool((err <= tol).all()), f"sequence {s} head {h}: {float((err / tol).max())} of the tolerance"
            if lse is not None:
                want = torch.logsumexp(z, -1)
                have = lse[at:at + n, h].double()
                assert bool((have[empty] == -math.inf).all())
                assert bool(((have - want).abs()[~empty] <= (2 * logit + 2.0 ** -20 * want.abs())[~empty]).all())
        at += n
    b.ok()


def _random_tree(n, rng):
    """Ancestor-or-self masks of n rows in breadth-first order, [n][2] words"""
    anc = np.zeros((n, 2), np.uint64)
    for i in range(n):
        if i:
            anc[i] = anc[int(rng.integers(max(0, i - 9), i))]
        anc[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return anc


HEADS = [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 14, 2, 128), ("fp32", 4, 2, 64), ("bf16", 3, 1, 32), ("fp32", 8, 1, 128), ("bf16", 32, 1, 64)]
SHAPES = [([1], [1]), ([1], [200]), ([1, 1, 1, 1, 1], [17, 128, 129, 1000, 1]), ([2], [2]), ([130], [130]), ([70, 1, 0, 33], [400, 77, 12, 33]),
          ([300], [1111]), ([5, 3], [3, 64]), ([1] * 40, [1 + 13 * i for i in range(40)])]


@pytest.mark.parametrize("heads", range(len(HEADS)))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("page,order", [(16, "head"), (24, "token"), (200, "head"), (5, "token")])
def test_attention(heads, shape, page, order):
    """Ragged batches of chunks and single tokens, one position to some hundred, pages that end inside every tile; tokens outside the sequences keep their rows;
    rows at positions below zero get zeros."""
    dtype, Hq, Hkv, D = HEADS[heads]
    n, kv = SHAPES[shape]
    b = Batch(n, kv, page, Hkv, D, dtype, order, seed=heads * 100 + shape, front=1, back=2, spare_columns=3)
    q = _randn(_gen(1), b.tokens, Hq, D, dtype=DT[dtype], scale=1.5)
    out, lse = _attention(b, q)
    _check_attention(b, q, out, lse)


@pytest.mark.parametrize("heads", range(len(HEADS)))
@pytest.mark.parametrize("window", [1, 7, 100, 128, 5000])
def test_attention_with_a_window(heads, window):
    dtype, Hq, Hkv, D = HEADS[heads]
    b = Batch([150, 1, 9, 1], [700, 300, 9, 1], 16, Hkv, D, dtype, seed=window, front=0, back=1)
    q = _randn(_gen(2), b.tokens, Hq, D, dtype=DT[dtype])
    out, lse = _attention(b, q, window=window)
    _check_attention(b, q, out, lse, window=window)


@pytest.mark.parametrize("heads", range(len(HEADS)))
@pytest.mark.parametrize("n,kv", [([1], [50]), ([68], [1068]), ([128], [128]), ([30, 128, 7, 64], [900, 333, 7, 65]), ([4], [2])])
def test_attention_of_draft_trees(heads, n, kv):
    """Ancestor masks; bits of rows that the block does not have are ignored; a row without bits and without cached positions sees nothing."""
    dtype, Hq, Hkv, D = HEADS[heads]
    rng = np.random.default_rng(sum(n))
    b = Batch(n, kv, 16, Hkv, D, dtype, seed=heads, front=2, back=0)
    anc = np.zeros((b.tokens, 2), np.uint64)
    at = b.front
    for m in n:
        anc[at:at + m] = _random_tree(m, rng)
        if m < 128:
            anc[at, 1] |= np.uint64(1) << np.uint64(63)
        if m > 3:
            anc[at + 2] = 0
        at += m
    q = _randn(_gen(3), b.tokens, Hq, D, dtype=DT[dtype])
    out, lse = _attention(b, q, anc=anc)
    _check_attention(b, q, out, lse, anc=anc)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,n,kv", [
    ("bf16", 8, 2, 128, 16, [1], [5000]), ("bf16", 8, 2, 128, 16, [1, 1, 1], [4099, 31, 900]), ("bf16", 8, 2, 128, 24, [200], [3001]), ("bf16", 4, 1, 64, 64, [64, 1, 500], [3000, 2999, 700]),
    ("bf16", 4, 4, 64, 8, [1, 1], [777, 2049]), ("fp32", 4, 2, 64, 16, [1, 90], [3000, 1500]), ("bf16", 8, 1, 32, 10, [3], [2000]), ("bf16", 16, 1, 128, 32, [1], [9000])])
@pytest.mark.parametrize("window", [0, 1025])
def test_every_visible_position_counts_once(dtype, Hq, Hkv, D, page, n, kv, window):
    """Queries of zero weigh every visible key alike, and value p is 1 in dim p mod D alone: an output is the share of the visible positions of that residue, so one
    position lost or counted twice changes it by D / n of itself (above the 3 * 2^-8 of the roundings for n up to 10000 D / 128), and lse is log n to 2^-21."""
    b = Batch(n, kv, page, Hkv, D, dtype, seed=7, fill=0.0)
    b.v.fill_(NAN)                                     # slots of no position hold anything
    b.k.fill_(NAN)
    for s in range(len(n)):
        pg, sl = b.slots(s)
        b.view(b.k)[pg, sl] = 1.0
        b.view(b.v)[pg, sl] = torch.eye(D, device="cuda").repeat(-(-kv[s] // D), 1)[:kv[s], None].expand(-1, Hkv, -1).to(DT[dtype])
    q = torch.zeros(b.tokens, Hq, D, device="cuda", dtype=DT[dtype])
    out, lse = _attention(b, q, window=window)
    at = 0
    for s, m in enumerate(n):
        see = torch.from_numpy(_visible(m, kv[s], window, None)).double().cuda()
        count = see @ torch.eye(D, device="cuda", dtype=torch.float64).repeat(-(-kv[s] // D), 1)[:kv[s]]
        ref = (count / see.sum(1, keepdim=True))[:, None]
        assert bool(((out[at:at + m].double() - ref).abs() <= 3 * HALF[dtype] * ref).all()), s
        assert bool(((lse[at:at + m].double() - see.sum(1, keepdim=True).log()).abs() <= 2.0 ** -20 * 10).all()), s
        at += m
    b.ok()


@pytest.mark.parametrize("D,page,n,kv", [(128, 64, [16, 9, 1, 3, 30], [32100, 29999, 16000, 1, 30]), (64, 16, [4] * 6, [30000 - 77 * i for i in range(6)])])
def test_a_few_tokens_over_long_caches(D, page, n, kv):
    """Tiles of few pairs whose chunks go through both sets of scores in turn (more than 32 chunks for every CTA), beside one of one position: every visible
    position counts once, the last and the first of every token included, and random values stay within the roundings."""
    Hq, Hkv = 16, 8
    b = Batch(n, kv, page, Hkv, D, "bf16", seed=3, fill=0.0)
    for s in range(len(n)):
        pg, sl = b.slots(s)
        b.view(b.v)[pg, sl] = torch.eye(D, device="cuda").repeat(-(-kv[s] // D), 1)[:kv[s], None].expand(-1, Hkv, -1).to(torch.bfloat16)
    q = torch.zeros(b.tokens, Hq, D, device="cuda", dtype=torch.bfloat16)
    out, lse = _attention(b, q)
    at = 0
    for s, m in enumerate(n):
        for i in range(m):
            t = kv[s] - m + i + 1
            if t <= 0:                      # padding
                assert bool((out[at + i] == 0).all())
                continue
            count = torch.bincount(torch.arange(t) % D, minlength=D).double().cuda() / t
            # a share is rounded once, 2^-8; a position more or less is D / t of it, 2^-7.9 at the longest
            assert bool(((out[at + i].double() - count).abs() <= 2.0 ** -8 * 1.01 * count).all())
            assert bool(((lse[at + i].double() - math.log(t)).abs() <= 2.0 ** -20 * 11).all())
        at += m
    b.k.copy_(_randn(_gen(8), *b.k.shape))
    b.v.copy_(_randn(_gen(9), *b.v.shape))
    q = _randn(_gen(10), *q.shape, dtype=torch.bfloat16, scale=1.5)
    out, lse = _attention(b, q)
    _check_attention(b, q, out, lse)
    again, _ = _attention(b, q)
    assert torch.equal(out, again)


@pytest.mark.parametrize("heads", range(len(HEADS)))
@pytest.mark.parametrize("kind", ["causal", "window", "tree"])
def test_what_a_token_does_not_see_does_not_reach_it(heads, kind):
    """Keys and values of later positions, of other branches, in front of the window and behind kv_len are NaN or infinite: the rows that do not see them have the
    values they have without them, the rows that see an infinite value have it in its dimension, and only there."""
    dtype, Hq, Hkv, D = HEADS[heads]
    n, kv, window = (60, 400, 0) if kind != "window" else (60, 400, 90)
    b = Batch([n], [kv], 16, Hkv, D, dtype, seed=11, fill=NAN)
    g = _gen(12)
    pg, sl = b.slots(0)
    b.view(b.k)[pg, sl] = _randn(g, kv, Hkv, D, dtype=DT[dtype])
    b.view(b.v)[pg, sl] = _randn(g, kv, Hkv, D, dtype=DT[dtype])
    q = _randn(g, n, Hq, D, dtype=DT[dtype])
    anc = None
    if kind == "tree":
        anc = _random_tree(n, np.random.default_rng(1))
        L = kv - n
        spoil = {L + 20: math.inf, L + 41: NAN, L + 59: -math.inf}
    elif kind == "window":
        spoil = {300: math.inf, 255: NAN, 390: -math.inf, 399: NAN}       # 300, 255: out of the last rows' windows
    else:
        spoil = {350: -math.inf, 399: NAN, 385: math.inf}
    clean, _ = _attention(b, q, anc=anc, window=window)
    for p, x in spoil.items():
        b.view(b.v)[pg[p], sl[p], :, p % D] = x
    spoiled, _ = _attention(b, q, anc=anc, window=window)
    see = _visible(n, kv, window, anc)
    want = clean.clone()
    for p, x in spoil.items():
        rows = torch.from_numpy(np.where(see[:, p])[0]).cuda()
        want[rows, :, p % D] = want[rows, :, p % D] + x
    assert torch.equal(torch.isnan(want), torch.isnan(spoiled))
    fine = torch.isfinite(want)
    assert torch.equal(want.isinf() * want.sign(), spoiled.isinf() * spoiled.sign()) or torch.equal(want[want.isinf()], spoiled[want.isinf()])
    assert torch.equal(want[fine], spoiled[fine])
    # a key that is no number: only who sees it is touched
    b.view(b.k)[pg[kv - 1], sl[kv - 1]] = NAN
    last, _ = _attention(b, q, anc=anc, window=window)
    blind = torch.from_numpy(~see[:, kv - 1]).cuda()
    assert torch.equal(torch.nan_to_num(last[blind], nan=123.0), torch.nan_to_num(spoiled[blind], nan=123.0))
    assert bool(torch.isnan(last[~blind]).all())
    b.ok()


@pytest.mark.parametrize("heads", range(len(HEADS)))
@pytest.mark.parametrize("window", [1, 33, 90])
def test_what_a_single_token_does_not_see_does_not_reach_it(heads, window):
    """Single tokens with a window: keys and values in front of it and behind kv_len are NaN or infinite, and nothing of that shows."""
    dtype, Hq, Hkv, D = HEADS[heads]
    b = Batch([1, 1, 1], [400, 97, 31], 16, Hkv, D, dtype, seed=11)
    q = _randn(_gen(13), 3, Hq, D, dtype=DT[dtype])
    clean, l0 = _attention(b, q, window=window)
    _check_attention(b, q, clean, l0, window=window)
    keep_k, keep_v = b.k.clone(), b.v.clone()
    b.k.fill_(NAN)
    b.v.fill_(math.inf)
    for s in range(3):
        pg, sl = (x[max(0, b.kv[s] - window):] for x in b.slots(s))
        b.view(b.k)[pg, sl], b.view(b.v)[pg, sl] = b.view(keep_k)[pg, sl], b.view(keep_v)[pg, sl]
    spoiled, l1 = _attention(b, q, window=window)
    assert torch.equal(clean, spoiled) and torch.equal(l0, l1)


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 33, 1, 64), ("bf16", 64, 1, 128), ("bf16", 40, 2, 128), ("fp32", 40, 1, 32), ("bf16", 16, 1, 64), ("bf16", 9, 1, 128)])
@pytest.mark.parametrize("n,kv", [([1, 1], [300, 5]), ([9, 2], [400, 2])])
def test_attention_of_many_heads_on_one(dtype, Hq, Hkv, D, n, kv):
    b = Batch(n, kv, 16, Hkv, D, dtype, seed=5)
    q = _randn(_gen(1), b.tokens, Hq, D, dtype=DT[dtype])
    out, lse = _attention(b, q)
    _check_attention(b, q, out, lse)


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 2), ("fp32", 1)])
def test_attention_and_append_of_very_many_sequences(dtype, n):
    """1300 sequences: more than the threads that deal them have at hand."""
    Hq, Hkv, D, B = 4, 2, 64, 1300
    kv = [2 + (7 * i) % 61 for i in range(B)]
    b = Batch([n] * B, kv, 16, Hkv, D, dtype, seed=5, back=1)
    x = _randn(_gen(2), b.tokens, Hq + 2 * Hkv, D, dtype=DT[dtype])
    P.esp_paged_append(b.cache, b.batch, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
    out, _ = _attention(b, x[:, :Hq])
    b.ok()
    k, v = torch.zeros(B, 64, Hkv, D, device="cuda", dtype=DT[dtype]), torch.zeros(B, 64, Hkv, D, device="cuda", dtype=DT[dtype])
    for s in range(B):
        k[s, :kv[s]], v[s, :kv[s]] = b.read(b.k, s), b.read(b.v, s)
    at = torch.tensor(kv, device="cuda")
    assert torch.equal(k[torch.arange(B, device="cuda"), at - 1], x[n - 1:n * B:n, Hq:Hq + Hkv])
    q = x[:n * B, :Hq].view(B, n, Hkv, Hq // Hkv, D).double()
    z = torch.einsum("bihgd,bjhd->bhgij", q, k.double()) * D ** -0.5
    see = torch.arange(64, device="cuda") < (at[:, None] - n + 1 + torch.arange(n, device="cuda"))[..., None]
    w = torch.softmax(z.masked_fill(~see[:, None, None], -math.inf), -1)
    ref = torch.einsum("bhgij,bjhd->bihgd", w, v.double()).reshape(n * B, Hq, D)
    mag = torch.einsum("bhgij,bjhd->bihgd", w, v.double().abs()).reshape(n * B, Hq, D)
    # the weight's rounding, twice the logit's error ((D + 8) 2^-24 of about 40 at most, 2^-21) and the output's own rounding
    tol = ((0 if dtype == "fp32" else HALF["bf16"]) + 2 * (72 * 40 * 2.0 ** -24 + 2.0 ** -20)) * mag * 1.01 + HALF[dtype] * 1.01 * ref.abs()
    assert bool(((out[:-1].double() - ref).abs() <= tol).all()) and bool((out[-1] == 7.0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [1, 40])
def test_attention_of_steep_logits(dtype, n):
    """Logits that grow along the keys by thousands, so that the maximum moves in every chunk, and with a scale of the caller's."""
    Hq, Hkv, D, kv = 4, 2, 64, 900
    b = Batch([n], [kv], 16, Hkv, D, dtype, seed=3)
    pg, sl = b.slots(0)
    ramp = torch.arange(kv, device="cuda", dtype=torch.float32) / kv
    b.view(b.k)[pg, sl] = (ramp[:, None, None] * 8 + 0.01 * _randn(_gen(4), kv, Hkv, D)).to(DT[dtype])
    q = (8 + 0.1 * _randn(_gen(5), n, Hq, D)).to(DT[dtype])
    for scale in (0.0, 1.0, 0.001):
        out, lse = _attention(b, q, scale=scale)
        _check_attention(b, q, out, lse, scale=scale)
    out, lse = _attention(b, -q)
    _check_attention(b, -q, out, lse)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("what", ["q offset", "q head stride", "cache offset", "cache stride", "out offset", "head-major q and out"])
def test_attention_of_strides_without_alignment(dtype, n, what):
    Hq, Hkv, D, page, kv = 8, 2, 64, 16, [333, 64]
    b = Batch([n, n], kv, page, Hkv, D, dtype, seed=8)
    g = _gen(6)
    q = _randn(g, b.tokens, Hq, D, dtype=DT[dtype])
    ref, _ = _attention(b, q)
    _check_attention(b, q, ref, None)

    def moved(x, offset=0, pad=0):
        flat = torch.full((x.numel() // x.shape[-1] * (x.shape[-1] + pad) + offset,), 3.0, device="cuda", dtype=x.dtype)
        rows = x.shape[-1] + pad
        strides = [int(np.prod(x.shape[i + 1:-1])) * rows for i in range(x.dim() - 1)] + [1]
        y = flat.as_strided(x.shape, strides, offset)
        y.copy_(x)
        return flat, y
    out = None
    if what == "q offset":
        q = moved(q, 1)[1]
    elif what == "q head stride":
        q = moved(q, 0, 1)[1]
    elif what == "cache offset":
        (_, b.k), (_, b.v) = moved(b.k, 3), moved(b.v, 3)
        b.cache = P.PagedCache(b.k, b.v)
    elif what == "cache stride":
        (_, b.k), (_, b.v) = moved(b.k, 0, 2), moved(b.v, 0, 2)
        b.cache = P.PagedCache(b.k, b.v)
    elif what == "out offset":
        flat, out = moved(torch.full_like(q, 7.0), 1, 3)
    else:
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
        out = torch.full((Hq, b.tokens, D), 7.0, device="cuda", dtype=DT[dtype]).transpose(0, 1)
    got, lse = _attention(b, q, out=out)
    _check_attention(b, q, got, lse)
    if what == "out offset":
        got.fill_(3.0)
        assert bool((flat == 3.0).all())


def test_values_between_keys_and_interleaved_pages():
    """One tensor [pages, 2, ...] that holds both, as some servers lay them out, with a page stride of its own."""
    kv = torch.randn(9, 2, 2, 16, 128, device="cuda").bfloat16()
    b = Batch([3, 1], [60, 64], 16, 2, 128, "bf16", seed=1)
    kv[:b.k.shape[0], 0], kv[:b.k.shape[0], 1] = b.k, b.v
    b.k, b.v = kv[:b.k.shape[0], 0], kv[:b.k.shape[0], 1]
    b.cache = P.PagedCache(b.k, b.v)
    q = _randn(_gen(6), 4, 4, 128, dtype=torch.bfloat16)
    out, lse = _attention(b, q)
    _check_attention(b, q, out, lse)


@pytest.mark.parametrize("n", [1, 50])
def test_descriptions_that_do_not_hold_together_are_recorded(n):
    """The kernels' own checks: a sequence whose numbers contradict each other is left out, a page number that there is not is never followed; the status word says so
    and stays until it is cleared, the other sequences have their results."""
    b = Batch([n, n, n], [100, 200, 300], 16, 2, 128, "bf16", seed=2)
    q = _randn(_gen(7), 3 * n, 8, 128, dtype=torch.bfloat16)
    k, v = (_randn(_gen(s), 3 * n, 2, 128, dtype=torch.bfloat16) for s in (1, 2))
    good, _ = _attention(b, q)
    b.ok()

    def bad(change):
        keep = b.q_start.clone(), b.kv_len.clone(), b.table_d.clone()
        change()
        k0, v0 = b.k.clone(), b.v.clone()
        out, _ = _attention(b, q)
        with pytest.raises(P.EspError) as e:
            P.esp_paged_status(b.batch)
        assert e.value.code == -5
        b.status.zero_()
        P.esp_paged_append(b.cache, b.batch, k, v)
        with pytest.raises(P.EspError):
            P.esp_paged_status(b.batch)
        b.status.zero_()
        b.k.copy_(k0)
        b.v.copy_(v0)
        for x, y in zip((b.q_start, b.kv_len, b.table_d), keep):
            x.copy_(y)
        return out
    out = bad(lambda: b.kv_len[1:2].fill_(b.table.shape[1] * 16 + 1))
    assert bool((out[n:2 * n] == 7.0).all()) and torch.equal(out[:n].isfinite(), good[:n].isfinite())
    out = bad(lambda: b.kv_len[1:2].fill_(-1))
    assert bool((out[n:2 * n] == 7.0).all())
    out = bad(lambda: b.q_start[3:].fill_(3 * n + 1))
    assert bool((out[2 * n:] == 7.0).all())
    out = bad(lambda: b.q_start[1:2].fill_(2 * n + 1))          # the first one has too many tokens, the second starts behind its end
    assert bool((out[:2 * n] == 7.0).all())
    for page in (-1, b.k.shape[0], 2 ** 31 - 1):
        bad(lambda: b.table_d[1, 12:13].fill_(page))
    got, _ = _attention(b, q)
    assert torch.equal(got, good)
    b.ok()


@pytest.mark.parametrize("n,kv", [([1, 1, 1], [3000, 10, 500]), ([40, 1, 300], [3000, 10, 500])])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_same_call_gives_the_same_bits(dtype, n, kv):
    b = Batch(n, kv, 16, 2, 128, dtype, seed=2)
    q = _randn(_gen(7), b.tokens, 8, 128, dtype=DT[dtype])
    first, l1 = _attention(b, q)
    for _ in range(3):
        again, l2 = _attention(b, q)
        assert torch.equal(first, again) and torch.equal(l1, l2)


@pytest.mark.parametrize("dtype,D,n,kv", [("bf16", 128, [1] * 8, [9000] * 8), ("bf16", 128, [600, 68], [4000, 9000]), ("bf16", 64, [3, 300], [16000, 5000]), ("fp32", 64, [1, 20], [5000, 900])])
def test_many_calls_behind_one_another(dtype, D, n, kv):
    """Three hundred calls without a pause, on inputs larger than what the GPU keeps on chip among them: no wait runs out, every call gives the same bits."""
    b = Batch(n, kv, 16, 8, D, dtype, seed=2)
    q = _randn(_gen(7), b.tokens, 32, D, dtype=DT[dtype])
    sc, nb = _scratch(32, D)
    first, wrong = torch.empty_like(q), torch.zeros((), dtype=torch.int64, device="cuda")
    P.esp_paged_attention(b.cache, b.batch, q, first, sc, nb)
    out = torch.empty_like(q)
    for _ in range(300):
        P.esp_paged_attention(b.cache, b.batch, q, out, sc, nb)
        wrong += (out != first).sum()
    assert int(wrong) == 0
    b.ok()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_bound_on_new_tokens_far_above_them(dtype):
    """max_new is a bound: 2^31 - 1 is one too."""
    b = Batch([1, 7], [100, 50], 16, 2, 64, dtype, seed=2)
    b.batch = P.PagedBatch(b.q_start, b.kv_len, b.table_d, 2 ** 31 - 1, b.status)
    q = _randn(_gen(7), b.tokens, 8, 64, dtype=DT[dtype])
    out, lse = _attention(b, q)
    _check_attention(b, q, out, lse)


@pytest.mark.parametrize("dtype,tokens,Hq,Hkv", [("bf16", 2200, 64, 1), ("bf16", 1100, 64, 2), ("fp32", 300, 64, 1)])
def test_more_work_than_is_counted(dtype, tokens, Hq, Hkv):
    """A table that names one page for 2^30 positions: more chunks than 32 bits count, or 2^31 and more over the KV heads.  Nothing is walked or written."""
    k = torch.zeros(1, Hkv, 1024, 64, device="cuda", dtype=DT[dtype])
    table = torch.zeros(1, 2 ** 20, device="cuda", dtype=torch.int32)
    status = torch.zeros(1, device="cuda", dtype=torch.int32)
    q_start = torch.tensor([0, tokens], device="cuda", dtype=torch.int32)
    kv_len = torch.tensor([2 ** 30], device="cuda", dtype=torch.int32)
    batch = P.PagedBatch(q_start, kv_len, table, tokens, status)
    q = torch.zeros(tokens, Hq, 64, device="cuda", dtype=DT[dtype])
    out = torch.full_like(q, 7.0)
    sc, nb = _scratch(Hq, 64)
    P.esp_paged_attention(P.PagedCache(k, k.clone()), batch, q, out, sc, nb)
    torch.cuda.synchronize()
    assert int(status) == 4 and bool((out == 7.0).all())


def test_nothing_to_do():
    b = Batch([0, 0], [5, 0], 16, 2, 128, "bf16", seed=2, front=2, back=1)
    q = _randn(_gen(7), 3, 8, 128, dtype=torch.bfloat16)
    out, lse = _attention(b, q)
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
    k0 = b.k.clone()
    P.esp_paged_append(b.cache, b.batch, q[:, :2], q[:, :2])
    assert torch.equal(b.k, k0)
    empty = torch.empty(0, 8, 128, device="cuda", dtype=torch.bfloat16)
    assert _attention(b, empty)[0].shape == (0, 8, 128)
    P.esp_paged_append(b.cache, b.batch, empty[:, :2], empty[:, :2], q=empty, q_out=torch.empty_like(empty))
    cfg = P.rope_cfg(128)
    P.esp_qk_norm_rope(empty, None, torch.empty_like(empty), None, cfg, _rope_table(cfg), torch.empty(0, dtype=torch.int32, device="cuda"))
    none = P.PagedBatch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
                        torch.empty(0, 4, dtype=torch.int32, device="cuda"), 1)
    sc, nb = _scratch(8, 128)
    P.esp_paged_attention(b.cache, none, q, out, sc, nb)
    assert bool((out == 7.0).all())
    b.ok()


# ================================================================ together, as a server runs them
def _layer(b, x, cfg, table, gains, positions=None, anc=None, window=0, stream=None, q_out=None, out=None, scratch=None):
    """Projection output -> pages and rotated queries -> attention"""
    Hkv = b.k.shape[1] if b.order == "head" else b.k.shape[2]
    Hq = x.shape[1] - 2 * Hkv
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    q_out = torch.empty(q.shape, device="cuda", dtype=x.dtype) if q_out is None else q_out
    P.esp_paged_append(b.cache, b.batch, k, v, cfg, table, positions=positions, k_gain=gains[1], q=q, q_out=q_out, q_gain=gains[0], stream=stream)
    out = torch.full(q.shape, 7.0, device="cuda", dtype=x.dtype) if out is None else out
    sc, nb = _scratch(Hq, x.shape[2]) if scratch is None else scratch
    P.esp_paged_attention(b.cache, b.batch, q_out, out, sc, nb, anc=anc, window=window, stream=stream)
    return q_out, out


@pytest.mark.parametrize("dtype,D,page,order", [("bf16", 128, 16, "head"), ("bf16", 64, 48, "token"), ("fp32", 64, 16, "token")])
def test_a_prompt_in_chunks_then_steps_then_a_tree(dtype, D, page, order):
    """A prompt of two sequences in uneven chunks, single tokens, then a draft tree: what stands in the pages and comes out is what the whole sequence in 64 bits gives,
    position by position; the keys in the pages are those of one call over the whole prompt, bit for bit."""
    Hq, Hkv = 8, 2
    lengths = [150, 71]
    b = Batch([0, 0], [170, 90], page, Hkv, D, dtype, order, seed=1, fill=NAN)
    g = _gen(2)
    cfg = P.rope_cfg(D, 10000.0)
    table = _rope_table(cfg)
    gains = [(1 + 0.1 * _randn(g, D)).to(DT[dtype]) for _ in range(2)]
    xs = [_randn(g, t + 20, Hq + 2 * Hkv, D, dtype=DT[dtype]) for t in lengths]
    done = [0, 0]

    def step(n, anc=None, positions=None):
        kv = [d + m for d, m in zip(done, n)]
        b.n, b.kv = n, kv
        b.q_start.copy_(torch.tensor([0, n[0], sum(n)], dtype=torch.int32))
        b.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        b.batch = P.PagedBatch(b.q_start, b.kv_len, b.table_d, max(n), b.status)
        x = torch.cat([xs[s][done[s]:kv[s]] for s in range(2)])
        q, out = _layer(b, x, cfg, table, gains, positions, None if anc is None else torch.from_numpy(anc.view(np.int64)).cuda())
        _check_attention(b, q, out, None, anc=anc)
        for s in range(2):
            done[s] = kv[s]
    for n in ([64, 1], [50, 70], [36, 0], [1, 1], [1, 0]):
        step(n)
    for s in range(2):
        one = torch.empty(done[s], Hkv, D, device="cuda", dtype=DT[dtype])
        P.esp_qk_norm_rope(None, xs[s][:done[s], Hq:Hq + Hkv], None, one, cfg, table, torch.arange(done[s], dtype=torch.int32, device="cuda"), k_gain=gains[1])
        assert torch.equal(b.read(b.k, s), one) and torch.equal(b.read(b.v, s), xs[s][:done[s], Hq + Hkv:])
    n = [12, 9]
    rng = np.random.default_rng(4)
    trees = [_random_tree(m, rng) for m in n]
    depth = [[bin(int(w[0])).count("1") - 1 for w in t] for t in trees]
    pos = torch.tensor([done[s] + d for s in range(2) for d in depth[s]], dtype=torch.int32, device="cuda")
    step(n, anc=np.concatenate(trees), positions=pos)


@pytest.mark.parametrize("n", [[1, 1, 1], [1, 60, 4]])
def test_captured_and_replayed(n):
    """A captured append and attention read lengths, tables and tensors as they are when it is replayed; two graphs share the scratch, one after the other."""
    Hq, Hkv, D = 8, 2, 128
    cfg = P.rope_cfg(D)
    table = _rope_table(cfg)
    g = _gen(3)
    scratch = _scratch(Hq, D)
    graphs = []
    for seed in (1, 2):
        b = Batch(n, [300, 200, 100], 16, Hkv, D, "bf16", seed=seed)
        x = _randn(g, b.tokens, Hq + 2 * Hkv, D, dtype=torch.bfloat16)
        q, out = torch.empty(b.tokens, Hq, D, device="cuda", dtype=torch.bfloat16), torch.full((b.tokens, Hq, D), 7.0, device="cuda", dtype=torch.bfloat16)
        _layer(b, x, cfg, table, [None, None], q_out=q, out=out, scratch=scratch)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _layer(b, x, cfg, table, [None, None], q_out=q, out=out, scratch=scratch, stream=torch.cuda.current_stream())
        graphs.append((graph, b, x, q, out))
    for kv in ([300, 200, 100], [17, 200, 64], [304, 61, 5]):
        for graph, b, x, q, out in graphs:
            b.kv = kv
            b.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
            x.copy_(_randn(g, *x.shape))
            out.fill_(7.0)
            graph.replay()
        torch.cuda.synchronize()
        for graph, b, x, q, out in graphs:
            _check_attention(b, q, out, None)


def test_on_another_stream_and_two_streams_at_once():
    """Calls on two streams, each with its own scratch, while both run."""
    Hq, Hkv, D = 8, 2, 128
    cfg = P.rope_cfg(D)
    table = _rope_table(cfg)
    runs = []
    for seed in (1, 2):
        b = Batch([1, 130, 2], [2000, 1500, 900], 16, Hkv, D, "bf16", seed=seed)
        runs.append((b, _randn(_gen(seed), b.tokens, Hq + 2 * Hkv, D, dtype=torch.bfloat16), torch.cuda.Stream(), _scratch(Hq, D), []))
    torch.cuda.synchronize()
    for _ in range(5):
        for b, x, stream, scratch, got in runs:
            with torch.cuda.stream(stream):
                got.append(_layer(b, x, cfg, table, [None, None], stream=stream, scratch=scratch))
    torch.cuda.synchronize()
    for b, x, stream, scratch, got in runs:
        for q, out in got:
            _check_attention(b, q, out, None)
            assert torch.equal(out, got[0][1])


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 elements (8.6 GB for keys, 8.6 for values): the pages at its far end."""
    Hq, Hkv, D, page = 8, 2, 128, 64
    n_pages = (1 << 32) // (Hkv * page * D) + 4
    k = torch.empty(n_pages, Hkv, page, D, device="cuda", dtype=torch.bfloat16)
    v = torch.empty_like(k)
    for n in (1, 100):
        b = Batch([n], [200], page, Hkv, D, "bf16", seed=1)
        far = [n_pages - 1, 0, n_pages - 3, 2]
        b.table = np.array([far], np.int32)
        b.table_d = torch.tensor(b.table, device="cuda")
        b.batch = P.PagedBatch(b.q_start, b.kv_len, b.table_d, n, b.status)
        b.k, b.v, b.cache = k, v, P.PagedCache(k, v)
        for p in far:
            k[p] = _randn(_gen(p % 1000), Hkv, page, D, dtype=torch.bfloat16)
            v[p] = _randn(_gen(p % 1000 + 1), Hkv, page, D, dtype=torch.bfloat16)
        x = _randn(_gen(5), n, Hq + 2 * Hkv, D, dtype=torch.bfloat16)
        q, out = _layer(b, x, None, None, [None, None])
        assert torch.equal(b.read(k, 0)[200 - n:], x[:, Hq:Hq + Hkv])
        _check_attention(b, q, out, None)
