"""Sampling (esp_sample) against its definition in 64 bits.

The kernel's sums are 64-bit ones of weights that are off by 2e-13 of themselves: a token may differ where uniform or top_p meets a border to 1e-11 of the sum, and only there.
"""
import math

import numpy as np
import pytest
import torch

import paper_2603_17942_b200 as P

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
NAN, INF = float("nan"), math.inf
NEAR = 1e-11


def _call(x, u, stream=None, logprob=True, **settings):
    rows, vocab = x.shape
    s = {k: None if v is None else torch.as_tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32).expand(rows).contiguous().cuda() for k, v in settings.items()}
    tokens, lp = torch.full((rows,), -7, dtype=torch.int32, device="cuda"), torch.full((rows,), 7.0, device="cuda") if logprob else None
    nb = P.esp_sample_scratch_bytes(rows, vocab)
    scratch = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")
    P.esp_sample(x, torch.as_tensor(u, dtype=torch.float32).expand(rows).contiguous().cuda(), tokens, scratch, nb, logprob=lp, stream=stream, **s)
    return tokens, lp


def _weights(x, t):
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    with np.errstate(invalid="ignore", over="ignore"):
        return x, np.where(x == top, 1.0, 0.0) if np.isinf(top) else np.where(np.isneginf(x), 0.0, np.exp((x - top) / t))


def _check_row(x, u, token, logprob, t=1.0, k=0, p=1.0, m=0.0):
    x = x.astype(np.float64)
    u, t, p, m = (np.float64(np.float32(v)) for v in (u, t, p, m))
    if not (t >= 0) or np.isinf(t) or not (u >= 0) or np.isnan(p) or np.isnan(m) or np.all(np.isnan(x) | np.isneginf(x)):
        assert token == -1 and math.isnan(logprob)
        return
    if t == 0:
        x, w = _weights(x, 1.0)
        k = 1
    else:
        x, w = _weights(x, t)
    order = np.argsort(-x, kind="stable")[:k if k > 0 else len(x)]
    mass = np.cumsum(w[order])
    fronts = [len(order)]
    if p < 1:
        before = np.concatenate([[0.0], mass[:-1]])
        fronts = sorted({max(1, int(np.searchsorted(before, p * mass[-1] * (1 + e) - 0.0, side="left"))) for e in (-NEAR, 0.0, NEAR)})
    least = min(m, 1.0)
    ok = []
    for front in fronts:
        kept = order[:front]
        kept = np.sort(kept[(w[kept] >= least) | (kept == order[0])])
        upto = np.cumsum(w[kept])
        total = upto[-1]
        at = np.where(kept == token)[0]
        if len(at) == 0 or w[token] == 0:
            continue
        lo, hi = upto[at[0]] - w[token], upto[at[0]]
        if lo - NEAR * total <= u * total < hi + NEAR * total or (u >= 1 and not (w[kept[at[0] + 1:]] > 0).any()):
            ok.append(abs(logprob - math.log(w[token] / total)) <= 2.0 ** -23 * (1 + abs(logprob)))        # fp32 of a logarithm of a quotient
    assert any(ok), (token, logprob, u, k, p, m, t, fronts)


def _check(x, u, tokens, lp, **settings):
    xs, tokens, lp = x.float().cpu().numpy(), tokens.cpu().numpy(), lp.cpu().numpy()
    u = np.broadcast_to(np.asarray(u, np.float32), len(xs))
    get = {k: np.broadcast_to(np.asarray(v, np.float64), len(xs)) for k, v in settings.items() if v is not None}
    for i in range(len(xs)):
        one = {a: get[b][i] for a, b in (("t", "temperature"), ("p", "top_p"), ("m", "min_p")) if b in get}
        _check_row(xs[i], u[i], int(tokens[i]), float(lp[i]), k=int(get["top_k"][i]) if "top_k" in get else 0, **one)


def _rows(rows, vocab, seed, dtype, kind):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, vocab, generator=g, device="cuda")
    if kind == "peaks":                       # a few tokens have most
        x = 2 * x
        few = max(1, min(48, vocab // 8))
        x.scatter_add_(1, torch.randint(0, vocab, (rows, few), generator=g, device="cuda"), 4 + 12 * torch.rand(rows, few, generator=g, device="cuda"))
    elif kind == "flat":                      # no one has
        x = 0.3 * x
    elif kind == "ties":                      # five values
        x = x.mul(1.2).round().clamp(-2, 2)
    elif kind == "equal":
        x = torch.zeros_like(x) - 3.25
    elif kind == "wide":                      # hardly two in a histogram
        x = 40 * x
    return x.to(DT[dtype])


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7), dict(top_k=1), dict(top_k=5), dict(top_k=50, temperature=0.8), dict(top_k=1900), dict(top_k=2500),
            dict(top_k=10 ** 6), dict(top_p=0.5), dict(top_p=0.9, temperature=0.6), dict(top_p=0.999), dict(top_p=0.0), dict(top_p=1e-9), dict(top_p=0.99999994),
            dict(min_p=0.05), dict(min_p=1e-6, temperature=1.3), dict(min_p=1.0), dict(min_p=7.0), dict(top_k=40, top_p=0.8), dict(top_k=3000, top_p=0.9, min_p=0.001),
            dict(top_p=0.95, min_p=0.02), dict(top_k=100, min_p=0.1), dict(top_k=30, top_p=0.9, min_p=0.02, temperature=1.1), dict(temperature=50.0), dict(temperature=1e-3),
            dict(temperature=1e-42), dict(temperature=3e38)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,kind", [(1, "normal"), (2, "normal"), (33, "peaks"), (500, "ties"), (4097, "normal"), (30011, "peaks"), (30011, "flat"), (30011, "ties"), (30011, "equal"),
                                        (30011, "wide"), (128256, "peaks"), (151936, "flat"), (262147, "peaks")])
def test_settings(dtype, vocab, kind):
    """Every combination of limits on every kind of row, uniform at both ends and between."""
    for i, settings in enumerate(SETTINGS):
        x = _rows(5, vocab, 7 * i + vocab, dtype, kind)
        u = np.array([0.0, 0.31, np.float32(np.random.default_rng(i).random()), 0.77, 1 - 2.0 ** -24], np.float32)
        tokens, lp = _call(x, u, **settings)
        _check(x, u, tokens, lp, **settings)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_row_has_its_own_settings(dtype):
    rows, vocab = 200, 5003
    x = _rows(rows, vocab, 3, dtype, "peaks")
    rng = np.random.default_rng(5)
    settings = dict(temperature=rng.choice([0.0, 0.5, 1.0, 2.0], rows), top_k=rng.choice([0, -3, 1, 20, 3000, vocab, vocab + 9], rows), top_p=rng.choice([0.3, 0.9, 1.0, 2.0], rows),
                    min_p=rng.choice([0.0, -1.0, 0.01, 0.3], rows))
    u = rng.random(rows, np.float32)
    tokens, lp = _call(x, u, **settings)
    _check(x, u, tokens, lp, **settings)
    again, lp2 = _call(x[17:19], u[17:19], **{k: v[17:19] for k, v in settings.items()})       # the same row gives the same token whoever is beside it
    assert torch.equal(again, tokens[17:19]) and torch.equal(lp2, lp[17:19])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_masked_infinite_and_undefined_logits(dtype):
    """Masks of -infinity and of the type's lowest value, rows that a mask leaves empty, NaN, +infinity; zeros of both signs are ties."""
    vocab, low = 6007, torch.finfo(DT[dtype]).min
    x = _rows(12, vocab, 4, dtype, "normal")
    x[0, 100:] = -INF
    x[1, 7:] = low
    x[2] = -INF
    x[3] = low
    x[4] = NAN
    x[5, ::2] = NAN
    x[6, [10, 4000]] = INF
    x[7] = INF
    x[8] = 0.0
    x[8, ::3] = -0.0
    x[9], x[9, 77] = -INF, -2.5
    x[10, ::2] = torch.finfo(DT[dtype]).max
    x[11] = x[11] * 1e-41 if dtype == "fp32" else x[11]
    for settings in (dict(), dict(temperature=0.0), dict(top_k=3), dict(top_k=2500), dict(top_p=0.6), dict(min_p=0.2), dict(top_k=6006, top_p=0.9), dict(temperature=1e38),
                     dict(temperature=3e38, top_p=0.5)):
        for u in (0.0, 0.4, 0.999999):
            tokens, lp = _call(x, u, **settings)
            _check(x, u, tokens, lp, **settings)
    tokens, _ = _call(x, 0.4, temperature=0.0)
    assert tokens[8] == 0 and tokens[6] == 10 and tokens[2] == -1 and tokens[4] == -1


def test_settings_that_mean_nothing():
    x = _rows(8, 3001, 4, "fp32", "normal")
    nan = NAN
    settings = dict(temperature=[nan, -1.0, INF, 1.0, 1.0, 1.0, 1.0, 1.0], top_p=[1.0, 1.0, 1.0, nan, 1.0, 1.0, 1.0, 0.9], min_p=[0.0, 0.0, 0.0, 0.0, nan, 0.0, 0.0, 0.0])
    u = np.array([0.5, 0.5, 0.5, 0.5, 0.5, nan, -0.1, 1.5], np.float32)
    tokens, lp = _call(x, u, **settings)
    assert tokens[:7].tolist() == [-1] * 7 and lp[:7].isnan().all()
    _check(x[7:], u[7:], tokens[7:], lp[7:], top_p=0.9)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,stride,offset", [(1000, 1003, 1), (1001, 1001, 0), (8000, 8192, 3), (777, 0, 0), (1, 1, 5)])
def test_strides_and_alignment(dtype, vocab, stride, offset):
    rows = 6
    flat = _rows(1, rows * max(stride, 1) + vocab + offset, 5, dtype, "normal")[0]
    x = flat[offset:].as_strided((rows, vocab), (stride, 1), flat.storage_offset() + offset)
    u = np.linspace(0.05, 0.95, rows).astype(np.float32)
    for settings in (dict(), dict(top_k=9, top_p=0.8)):
        tokens, lp = _call(x, u, **settings)
        _check(x, u, tokens, lp, **settings)
    assert torch.equal(_call(x, u, logprob=False, top_k=9, top_p=0.8)[0], tokens)


def test_shares_of_many_draws():
    """The tokens of 60000 uniform numbers have the shares of the distribution: chi-square with the kept tokens' degrees of freedom, within five standard deviations of its mean."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n, x = 60000, 2 * torch.randn(1, 40, generator=g, device="cuda")
    u = torch.rand(n, generator=g, device="cuda")
    tokens = _call(x.expand(n, 40), u, temperature=0.9, top_k=12)[0]
    p = torch.softmax(x[0].double() / np.float32(0.9), 0)
    keep = p.argsort(descending=True)[:12]
    p = p[keep] / p[keep].sum()
    count = torch.bincount(tokens.long(), minlength=40)
    assert count.sum() == count[keep].sum() == n
    chi = float(((count[keep] - n * p) ** 2 / (n * p)).sum())
    assert abs(chi - 11) < 5 * math.sqrt(22)


def test_the_vocabulary_that_no_block_keeps():
    """More logits than the shared memory of a cluster holds."""
    vocab = 700001
    for dtype in ("fp32", "bf16"):
        x = _rows(2, vocab, 9, dtype, "normal")
        for settings in (dict(), dict(top_k=60), dict(top_k=5000, top_p=0.9), dict(top_p=0.7), dict(min_p=0.3)):
            tokens, lp = _call(x, [0.2, 0.9], **settings)
            _check(x, np.array([0.2, 0.9], np.float32), tokens, lp, **settings)


@pytest.mark.parametrize("dtype,rows,vocab", [("fp32", 60, 30011), ("bf16", 60, 30011), ("fp32", 3, 2 ** 21), ("bf16", 2, 2 ** 21)])
def test_long_fronts(dtype, rows, vocab):
    """Nuclei of thousands of tokens, more rows of them than there are clusters for; logits far from zero, temperatures that make a bin of logits wide or narrow."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    u = np.random.default_rng(vocab).random(rows).astype(np.float32)
    p = np.linspace(0.6, 0.9999, rows)
    for scale, offset, t in ((1.0, 0.0, 1.0), (3.0, -200.0, 4.0), (0.01, 7.0, 0.01), (1e5, 0.0, 9e4), (30.0, 1e6, 50.0), (1e9, 3e9, 1e9), (1e-4, 0.0, 1e-4), (1.0, 0.0, 20.0)):
        x = (scale * torch.randn(rows, vocab, generator=g, device="cuda") + offset).to(DT[dtype])
        settings = dict(top_p=p, temperature=t)
        tokens, lp = _call(x, u, **settings)
        _check(x, u, tokens, lp, **settings)


def test_streams_and_graphs():
    x = _rows(20, 20011, 6, "bf16", "peaks")
    u = torch.rand(20, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    want, lp = _call(x, u, top_p=0.9)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got, _ = _call(x, u, stream=side, top_p=0.9)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    tokens, p = torch.empty_like(want), torch.full((20,), 0.9, device="cuda")
    nb = P.esp_sample_scratch_bytes(20, 20011)
    scratch = torch.empty(nb, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.esp_sample(x, u, tokens, scratch, nb, top_p=p)
    x.copy_(_rows(20, 20011, 8, "bf16", "peaks"))
    p.fill_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(tokens, _call(x, u, top_p=0.5)[0])
