"""The attention that cached positions receive (esp_paged_key_weights), against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_gpu_paged import DT, NAN, Batch, _gen, _randn
from tests.test_gpu_paged import _scratch as _attention_scratch

pytestmark = pytest.mark.gpu


class Scores:
    """Numbers for every slot, with strides of their own: gap elements between rows hold a mark."""

    def __init__(self, b, fill=None, seed=1, gap=0, dtype=torch.float32):
        shape = list(b.k.shape[:3])
        self.flat = torch.full((shape[0], shape[1], shape[2] + gap), -77, dtype=dtype, device="cuda")
        self.x = self.flat[..., :shape[2]]
        if fill is not None:
            self.x.fill_(fill)
        else:
            self.x.copy_(torch.rand(shape, generator=_gen(seed), device="cuda"))
        self.slots = P.PagedSlots(self.x, order=b.order)

    def view(self, b, x=None):
        x = self.x if x is None else x
        return x if b.order == "token" else x.transpose(1, 2)             # [page, slot, head]


def _visible(b, s, window, anc, last):
    """[observed tokens, kv] of what they see, and the first observed token."""
    n, t = b.n[s], b.kv[s]
    L, i0 = t - n, max(0, n - last) if last else 0
    i, j = torch.arange(i0, n, device="cuda")[:, None], torch.arange(t, device="cuda")[None]
    if anc is None:
        seen = j <= L + i
        if window:
            seen = seen & (j > L + i - window)
    else:
        at = b.front + sum(b.n[:s])
        bits = anc[at + i0:at + n].cpu().tolist()
        rows = torch.tensor([[bool((((lo & (2 ** 64 - 1)) | ((hi & (2 ** 64 - 1)) << 64)) >> c) & 1) for c in range(n)] for lo, hi in bits], device="cuda").view(n - i0, n)
        tree = torch.zeros(n - i0, t, dtype=torch.bool, device="cuda")
        c0 = max(0, -L)
        tree[:, max(L, 0):] = rows[:, c0:c0 + t - max(L, 0)]
        seen = (j < L) | tree
    return seen & (L + i >= 0), i0


def _logits(b, q, s):
    at = b.front + sum(b.n[:s])
    k = b.read(b.k, s).double()                                                             # [kv, Hkv, D]
    g = q.shape[1] // k.shape[1]
    x = q[at:at + b.n[s]].double().view(b.n[s], k.shape[1], g, -1)
    d = k.shape[2]
    return torch.einsum("ihgd,jhd->ihgj", x, k) / math.sqrt(d), torch.einsum("ihgd,jhd->ihgj", x.abs(), k.abs()) / math.sqrt(d)


def _lse(b, q, window=0, anc=None):
    out = torch.full((b.tokens, q.shape[1]), NAN, device="cuda")
    for s in range(len(b.n)):
        if b.n[s] == 0:
            continue
        at = b.front + sum(b.n[:s])
        seen, _ = _visible(b, s, window, anc, 0)
        x = _logits(b, q, s)[0].masked_fill(~seen[:, None, None], -math.inf)
        out[at:at + b.n[s]] = torch.logsumexp(x, -1).flatten(1).float() if b.kv[s] else -math.inf
    return out


def _check(b, q, lse, before, scores, keep, window=0, anc=None, last=0):
    """A weight's exponent is off by the product's sum, D roundings of the sum of magnitudes at most (twice that where the tensor cores cut off), three roundings of scale, score and
    lse and one of their difference; the exponential by 2^-22; the sum over P weights, all positive, by P + 4 roundings; keep * old + sum by two."""
    want, tol = before.double(), torch.zeros_like(before, dtype=torch.float64)
    view, tview = scores.view(b, want), scores.view(b, tol)
    for s in range(len(b.n)):
        n, t = b.n[s], b.kv[s]
        if n == 0 or t == 0:
            continue
        at, (page, slot) = b.front + sum(b.n[:s]), b.slots(s)
        seen, i0 = _visible(b, s, window, anc, last)
        x, size = (y[i0:] for y in _logits(b, q, s))
        l = lse[at + i0:at + n].double().view(n - i0, x.shape[1], x.shape[2])[..., None]
        w = torch.where(seen[:, None, None], (x - l).exp(), 0.0)
        rel = (q.shape[2] * size * 2.0 ** -23 + 4 * 2.0 ** -24 * (x.abs() + l.abs().nan_to_num(0, 0, 0)) + 2.0 ** -21)
        terms = (n - i0) * x.shape[2]
        total, err = w.sum((0, 2)), torch.where(seen[:, None, None], w * rel, 0.0).sum((0, 2))     # [Hkv, kv]
        old = torch.where(torch.arange(t, device="cuda") < t - n, keep * view[page, slot].T, 0.0) if keep else torch.zeros_like(total)
        view[page, slot] = (total + old).T
        tview[page, slot] = (err + (terms + 4) * 2.0 ** -24 * total + 2.0 ** -23 * (total + old.abs()) + 1e-30).T
    got = scores.x.double()
    assert torch.equal(got.isnan(), want.isnan())
    bad = (got - want).abs().nan_to_num(0) - tol
    assert (bad <= 0).all(), f"worst {float((bad + tol).max())}, of its tolerance {float(((bad + tol) / (tol + 1e-300)).max())}"
    if scores.flat.shape[2] > scores.x.shape[2]:
        assert (scores.flat[..., scores.x.shape[2]:] == -77).all()


def _scratch(b, q):
    nb = P.esp_paged_key_weights_scratch_bytes(b.tokens, q.shape[1], q.shape[2])
    return torch.full((nb,), 255, dtype=torch.uint8, device="cuda"), nb                    # NaN everywhere: contents are of no account


def _run(b, q, keep=1.0, window=0, anc=None, last=0, gap=0, lse=None, fill=None):
    lse = _lse(b, q, window, anc) if lse is None else lse
    scores = Scores(b, gap=gap, fill=fill)
    before = scores.x.clone()
    P.esp_paged_key_weights(b.cache, b.batch, q, lse, scores.slots, *_scratch(b, q), anc=anc, window=window, last=last, keep=keep)
    _check(b, q, lse, before, scores, keep, window, anc, last)
    b.ok()
    return scores, lse


SHAPES = [([1], [1]), ([1], [33]), ([1], [5000]), ([1] * 70, list(range(1, 71))), ([5, 1, 0, 130], [5, 300, 40, 200]), ([3, 4], [1, 9]), ([300], [900]), ([2, 1, 2], [2000, 64, 257]),
          ([40, 7], [40, 1031])]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,order", [("bf16", 8, 2, 128, 16, "head"), ("bf16", 14, 2, 128, 64, "token"), ("bf16", 16, 1, 64, 24, "token"), ("bf16", 3, 3, 64, 200, "head"),
                                                       ("bf16", 64, 1, 128, 8, "head"), ("bf16", 8, 2, 128, 17, "head"), ("bf16", 4, 2, 32, 16, "token"),
                                                       ("fp32", 4, 2, 64, 16, "head"), ("fp32", 6, 1, 128, 7, "token"), ("fp32", 40, 1, 32, 32, "head")])
@pytest.mark.parametrize("n,kv", SHAPES)
@pytest.mark.parametrize("keep", [0.0, 0.75])
def test_causal(dtype, Hq, Hkv, D, page, order, n, kv, keep):
    """Types, groups, head sizes, page sizes and orders; single tokens, prompts, padding, many sequences, one with no new token.  Other slots keep their bits."""
    b = Batch(n, kv, page, Hkv, D, dtype, order, seed=sum(kv) + D, front=2, back=3)
    q = _randn(_gen(3), b.tokens, Hq, D, dtype=DT[dtype], scale=2.0)
    _run(b, q, keep, gap=3)


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 14, 2, 64), ("fp32", 8, 2, 64), ("bf16", 8, 2, 32)])
@pytest.mark.parametrize("n,kv", [([1, 1], [700, 30]), ([5, 130], [600, 400]), ([3, 4], [1, 9])])
@pytest.mark.parametrize("window,last", [(1, 0), (33, 0), (300, 0), (0, 1), (0, 7), (0, 1000), (90, 3), (2 ** 30, 0)])
def test_windows_and_observed_tokens(dtype, Hq, Hkv, D, n, kv, window, last):
    b = Batch(n, kv, 16, Hkv, D, dtype, seed=window + last)
    q = _randn(_gen(4), b.tokens, Hq, D, dtype=DT[dtype])
    _run(b, q, 1.0, window=window if window < 2 ** 20 else 2 ** 30, last=last)


def _trees(b, seed):
    """Random masks: each row itself and some rows of its block, a row with none, bits of rows that the block does not have."""
    g = _gen(seed)
    anc = torch.randint(-2 ** 63, 2 ** 63 - 1, (b.tokens, 2), generator=g, device="cuda")
    anc[b.front + b.n[0] - 1] = 0
    return anc


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 14, 2, 64), ("bf16", 4, 4, 64), ("fp32", 8, 2, 64), ("bf16", 8, 2, 32)])
@pytest.mark.parametrize("n,kv", [([6], [6]), ([68, 1, 128], [300, 40, 700]), ([5, 9], [3, 600]), ([2, 3], [270, 65])])
@pytest.mark.parametrize("last", [0, 2])
def test_trees(dtype, Hq, Hkv, D, n, kv, last):
    b = Batch(n, kv, 16, Hkv, D, dtype, seed=sum(n), front=1)
    q = _randn(_gen(5), b.tokens, Hq, D, dtype=DT[dtype])
    _run(b, q, 0.5, anc=_trees(b, 6), last=last)


@pytest.mark.parametrize("Hq,Hkv,D,page,pad", [(8, 2, 128, 17, 0), (14, 2, 64, 9, 0), (40, 1, 128, 5, 0), (64, 1, 64, 17, 2), (3, 3, 128, 1, 0), (28, 4, 128, 16, 2), (6, 2, 64, 24, 4)])
@pytest.mark.parametrize("n,kv", [([1, 1, 1], [700, 30, 1]), ([5, 130, 2], [600, 400, 1000]), ([60], [61])])
@pytest.mark.parametrize("window,last,tree", [(0, 0, False), (33, 0, False), (300, 40, False), (0, 3, False), (0, 0, True), (0, 9, True)])
def test_rows_that_no_box_fits(Hq, Hkv, D, page, pad, n, kv, window, last, tree):
    """bf16 in pages that are no whole eights of slots, and queries whose heads do not lie on 16 bytes; passes that end inside a token's group of heads."""
    if tree and max(n) > 128:
        n = [min(x, 128) for x in n]
    b = Batch(n, kv, page, Hkv, D, "bf16", "token" if page % 2 else "head", seed=window + last + D, front=1)
    q = _randn(_gen(4), b.tokens, Hq, D + pad, dtype=DT["bf16"])[..., :D]
    _run(b, q, 0.9, window=window, last=last, anc=_trees(b, 6) if tree else None)


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 32, 2, 64), ("fp32", 8, 2, 64)])
@pytest.mark.parametrize("n,kv,window", [([1, 1], [900, 300], 0), ([40, 3], [900, 300], 0), ([1, 70], [1000, 1000], 130)])
def test_with_the_lse_of_the_attention(dtype, Hq, Hkv, D, n, kv, window):
    """Together with esp_paged_attention: a query head's weights add up to 1.  (Its lse is off by a few 2^-22 of its magnitude, below 16 here: 2^-17 of a weight covers it.)"""
    b = Batch(n, kv, 16, Hkv, D, dtype, seed=5)
    q = _randn(_gen(8), b.tokens, Hq, D, dtype=DT[dtype], scale=2.0)
    lse = torch.empty(b.tokens, Hq, device="cuda")
    P.esp_paged_attention(b.cache, b.batch, q, torch.empty_like(q), *_attention_scratch(Hq, D), window=window, lse=lse)
    scores, _ = _run(b, q, 0.0, window=window, lse=lse, fill=0.0)
    total = scores.view(b)
    for s in range(len(n)):
        page, slot = b.slots(s)
        assert torch.allclose(total[page, slot].double().sum(0), torch.full((Hkv,), float(n[s] * Hq // Hkv), dtype=torch.float64, device="cuda"), rtol=2.0 ** -15)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,n,kv", [("bf16", 8, 2, 128, [1, 1], [300, 65]), ("bf16", 8, 2, 128, [70, 9], [300, 65]), ("bf16", 8, 2, 64, [3], [100]),
                                                 ("fp32", 8, 2, 64, [70, 9], [300, 65])])
def test_what_is_not_seen_does_not_matter(dtype, Hq, Hkv, D, n, kv):
    """NaN in slots behind kv_len, in scores of new tokens and, with keep 0, in all; NaN in keys behind every window; queries and lse of unobserved tokens."""
    b = Batch(n, kv, 24, Hkv, D, dtype, seed=11)
    q = _randn(_gen(9), b.tokens, Hq, D, dtype=DT[dtype])
    window, last = 40, 2
    lse = _lse(b, q, window)
    clean, _ = _run(b, q, 0.0, window=window, last=last, lse=lse)
    behind = torch.ones(b.k.shape[:3], dtype=torch.bool, device="cuda")
    mark = behind if b.order == "token" else behind.transpose(1, 2)
    for s in range(len(n)):
        page, slot = b.slots(s)
        lo = max(0, kv[s] - min(last, n[s]) - window + 1)
        mark[page[lo:], slot[lo:]] = False
    b.k[behind] = NAN
    at = 0
    for m in n:
        q[at:at + max(0, m - last)] = NAN
        lse[at:at + max(0, m - last)] = NAN
        at += m
    scores = Scores(b, fill=NAN)
    P.esp_paged_key_weights(b.cache, b.batch, q, lse, scores.slots, *_scratch(b, q), window=window, last=last, keep=0.0)
    b.ok()
    for s in range(len(n)):
        page, slot = b.slots(s)
        assert torch.equal(scores.view(b)[page, slot], clean.view(b)[page, slot])


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 50), ("fp32", 5)])
def test_undefined_numbers_reach_what_sees_them(dtype, n):
    b = Batch([n, n], [200, 100], 16, 2, 64, dtype, seed=2)
    q = _randn(_gen(9), b.tokens, 8, 64, dtype=DT[dtype])
    lse = _lse(b, q)
    clean, _ = _run(b, q, 0.0, lse=lse)
    lse[n - 1, 5] = NAN                                             # the last token of the first sequence, KV head 1
    page, slot = b.slots(1)
    b.view(b.k)[page[10], slot[10], 0] = NAN                        # a key of the second sequence, KV head 0
    scores = Scores(b, fill=0.0)
    P.esp_paged_key_weights(b.cache, b.batch, q, lse, scores.slots, *_scratch(b, q), keep=0.0)
    b.ok()
    got, want = scores.view(b), clean.view(b)
    p0, s0 = b.slots(0)
    assert got[p0, s0][:, 1].isnan().all() and torch.equal(got[p0, s0][:, 0], want[p0, s0][:, 0])
    nan = got[page, slot].isnan()
    assert nan[10, 0] and nan.sum() == 1 and torch.equal(got[page, slot][~nan], want[page, slot][~nan])


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 60), ("fp32", 9)])
def test_pages_behind_the_window_may_be_gone(dtype, n):
    """Entries that name no page and that no observed token sees are passed over; one that is seen is recorded."""
    b = Batch([n], [500], 16, 2, 64, dtype, seed=3)
    q = _randn(_gen(1), b.tokens, 4, 64, dtype=DT[dtype])
    lse = _lse(b, q, 100)
    clean, _ = _run(b, q, 0.0, window=100, lse=lse)
    gone = (500 - n - 99) // 16
    b.table_d[0, :gone] = torch.tensor([-1, 10 ** 6], dtype=torch.int32, device="cuda").repeat(gone)[:gone]
    scores = Scores(b, fill=-3.0)
    P.esp_paged_key_weights(b.cache, b.batch, q, lse, scores.slots, *_scratch(b, q), window=100, keep=0.0)
    b.ok()
    page, slot = b.slots(0)
    assert (scores.view(b)[page[:gone * 16], slot[:gone * 16]] == -3.0).all()
    assert torch.equal(scores.view(b)[page[gone * 16:], slot[gone * 16:]], clean.view(b)[page[gone * 16:], slot[gone * 16:]])
    b.table_d[0, 31] = -1
    P.esp_paged_key_weights(b.cache, b.batch, q, lse, scores.slots, *_scratch(b, q), window=100, keep=0.0)
    with pytest.raises(P.EspError):
        b.ok()


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 20), ("fp32", 2)])
def test_sequences_that_do_not_hold_together(dtype, n):
    """They are left out and recorded, the others have their results."""
    b = Batch([n] * 4, [100, 200, 300, 64], 16, 2, 64, dtype, seed=3)
    q = _randn(_gen(1), b.tokens, 4, 64, dtype=DT[dtype])
    lse = _lse(b, q)
    clean, _ = _run(b, q, 0.0, lse=lse)
    for change in ("kv", "kv high", "q"):
        kv, start = b.kv_len.clone(), b.q_start.clone()
        if change == "kv":
            kv[1] = -4
        elif change == "kv high":
            kv[1] = 2 ** 30
        else:
            start[1] = 3 * n                                         # the second begins behind where it ends: neither it nor the first, which is too long, holds together
        batch = P.PagedBatch(start, kv, b.table_d, n, b.status)
        scores = Scores(b, fill=-3.0)
        P.esp_paged_key_weights(b.cache, batch, q, lse, scores.slots, *_scratch(b, q), keep=0.0)
        with pytest.raises(P.EspError):
            b.ok()
        b.status.zero_()
        for s in range(4):
            page, slot = b.slots(s)
            out = s == 1 or (change == "q" and s == 0)
            got = scores.view(b)[page, slot]
            assert torch.equal(got, torch.full_like(got, -3.0) if out else clean.view(b)[page, slot]), (change, s)


@pytest.mark.parametrize("dtype,n,kv", [("bf16", [1] * 40, [900] * 40), ("bf16", [400, 30], [900, 5000]), ("fp32", [60], [700])])
def test_the_same_call_gives_the_same_bits_on_another_stream_and_in_a_graph(dtype, n, kv):
    b = Batch(n, kv, 16, 2, 64, dtype, seed=7)
    q = _randn(_gen(1), b.tokens, 8, 64, dtype=DT[dtype])
    want, lse = _run(b, q, 0.0)
    side, scratch = torch.cuda.Stream(), _scratch(b, q)
    scores = Scores(b)
    for _ in range(3):
        scores.x.copy_(Scores(b).x)
        torch.cuda.synchronize()
        P.esp_paged_key_weights(b.cache, b.batch, q, lse, scores.slots, *scratch, keep=0.0, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(scores.x, want.x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.esp_paged_key_weights(b.cache, b.batch, q, lse, scores.slots, *scratch, keep=0.0)
    # a replay reads lengths and tensors as they are then
    kv2 = [max(1, t - 5) if m == 1 else t for m, t in zip(n, kv)]
    b.kv_len.copy_(torch.tensor(kv2, dtype=torch.int32))
    b.kv = kv2
    lse.copy_(_lse(b, q))
    scores.x.copy_(Scores(b).x)
    before = scores.x.clone()
    graph.replay()
    torch.cuda.synchronize()
    _check(b, q, lse, before, scores, 0.0)
