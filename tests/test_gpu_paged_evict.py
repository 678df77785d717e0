"""Cutting caches to budgets (esp_paged_evict) and accepting draft trees (esp_paged_accept): whole numbers and moved rows, equal bit by bit to plain loops."""
import math

import numpy as np
import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_gpu_key_weights import Scores
from tests.test_gpu_paged import DT, NAN, Batch, _gen, _randn

pytestmark = pytest.mark.gpu
INF = math.inf


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _reference(b, x, budget, recent, pos=None, settled=None, seen=None, left=()):
    """Everything that a call writes, from the definition: (k, v, scores, positions, settled, kv_len)."""
    Hkv = b.cache.c.n_kv_heads
    k, v, x = b.view(b.k).clone(), b.view(b.v).clone(), x.clone()
    pos = None if pos is None else pos.clone()
    settled_out, kv_out = None if settled is None else list(settled), list(b.kv)
    for s, t in enumerate(b.kv):
        keep = budget[s]
        if t <= keep or s in left:
            continue
        kv_out[s] = keep
        page, slot = b.slots(s)
        for h in range(Hkv):
            score = x[page, slot, h].double().cpu().numpy()
            where = np.arange(t) if pos is None else np.where(np.arange(t) < settled[s], pos[page, slot, h].cpu().numpy(), seen[s] - t + np.arange(t))
            now = t if pos is None else seen[s]
            rank = np.where(where >= now - recent, np.inf, np.where(np.isnan(score), -np.inf, score))
            best = np.zeros(t, bool)
            best[np.lexsort((np.arange(t), -rank))[:keep]] = True
            source, target = np.nonzero(best[keep:])[0] + keep, np.nonzero(~best[:keep])[0]
            assert len(source) == len(target)
            if pos is not None:
                pos[page[:keep], slot[:keep], h] = torch.tensor(where[:keep].astype(np.int32), device="cuda")
                pos[page[target], slot[target], h] = torch.tensor(where[source].astype(np.int32), device="cuda")
            for y in (k, v, x):
                y[page[target], slot[target], h] = y[page[source], slot[source], h]
        if settled is not None:
            settled_out[s] = keep
    return k, v, x, pos, settled_out, kv_out


def _same(a, b):
    return torch.equal(a.contiguous().view(torch.int16 if a.element_size() == 2 else torch.int32), b.contiguous().view(torch.int16 if b.element_size() == 2 else torch.int32))


def _scratch(b, max_kv=None):
    nb = P.esp_paged_evict_scratch_bytes(len(b.kv), b.cache.c.n_kv_heads, max(b.kv) if max_kv is None else max_kv)
    return torch.full((nb,), 255, dtype=torch.uint8, device="cuda"), nb


def _cut(b, scores, budget, recent=0, positions=None, settled=None, seen=None, stream=None, in_place=False, scratch=None, left=()):
    want = _reference(b, scores.view(b), budget, recent, None if positions is None else positions.view(b), settled, seen, left)
    settled_d, seen_d = (None if y is None else _i32(y) for y in (settled, seen))
    out = b.kv_len if in_place else torch.full_like(b.kv_len, -9)
    P.esp_paged_evict(b.cache, b.batch, scores.slots, _i32(budget), out, *(scratch or _scratch(b)), recent=recent, positions=None if positions is None else positions.slots,
                      settled=settled_d, seen=seen_d, stream=stream)
    torch.cuda.synchronize()
    assert out.tolist() == want[5]
    assert _same(b.view(b.k), want[0]) and _same(b.view(b.v), want[1]) and _same(scores.view(b), want[2])
    if positions is not None:
        assert torch.equal(positions.view(b), want[3]) and settled_d.tolist() == want[4]
    for y in (scores, positions):
        if y is not None and y.flat.shape[2] > y.x.shape[2]:
            assert (y.flat[..., y.x.shape[2]:] == -77).all()
    return want


def _batch(kv, page, Hkv, D, dtype, order, seed, **kw):
    return Batch([1 if t else 0 for t in kv], kv, page, Hkv, D, dtype, order, seed=seed, **kw)


LENGTHS = [([1], [0]), ([1], [1]), ([2], [1]), ([33, 0, 5], [32, 0, 9]), ([5, 300, 40, 200], [7, 100, 39, 1]), ([1000, 1025], [999, 24]), ([4097, 900], [4096, 64]), ([9000], [4500]),
           ([100] * 40, list(range(70, 110)))]


@pytest.mark.parametrize("dtype,Hkv,D,page,order", [("bf16", 2, 128, 16, "head"), ("bf16", 8, 64, 24, "token"), ("fp32", 3, 64, 17, "head"), ("fp32", 1, 32, 200, "token"),
                                                    ("bf16", 1, 32, 1, "head"), ("fp32", 2, 128, 64, "token")])
@pytest.mark.parametrize("kv,budget", LENGTHS)
@pytest.mark.parametrize("kind", ["wide", "ties", "odd"])
def test_cut(dtype, Hkv, D, page, order, kv, budget, kind):
    """Scores that all differ, many equal ones, zeros of both signs, infinities and NaN; with the latest ones held and without.  Slots that do not move keep their bits."""
    b = _batch(kv, page, Hkv, D, dtype, order, seed=sum(kv) + D)
    for recent in (0, min(budget) // 2):
        scores = Scores(b, seed=3, gap=2)
        if kind == "ties":
            scores.x.copy_((scores.x * 4).floor())
        elif kind == "odd":
            pick = torch.randint(0, 9, scores.x.shape, generator=_gen(4), device="cuda")
            for i, y in enumerate((0.0, -0.0, INF, -INF, NAN, -3.0)):
                scores.x[pick == i] = y
        _cut(b, scores, budget, recent)
        b.ok()


@pytest.mark.parametrize("dtype,D,order", [("bf16", 64, "head"), ("fp32", 64, "token")])
@pytest.mark.parametrize("recent", [0, 1, 30])
def test_positions_through_several_cuts(dtype, D, order, recent):
    """A server's use: tokens are appended behind the settled slots, the cache is cut again and again; the latest positions always stay, whatever their scores."""
    Hkv, budgets = 2, [60, 100, 64]
    kv, settled, seen = [150, 90, 64], [0, 0, 0], [150, 90, 64]
    b = _batch([200] * 3, 16, Hkv, D, dtype, order, seed=6)
    scores, positions = Scores(b, seed=1, gap=1), Scores(b, fill=-5, gap=1, dtype=torch.int32)
    for step in range(5):
        b.kv = kv
        b.kv_len.copy_(_i32(kv))
        scores.x.copy_(torch.rand(scores.x.shape, generator=_gen(step), device="cuda"))
        _, _, _, _, settled, kv = _cut(b, scores, budgets, recent, positions, settled, seen)
        for s in range(3):
            page, slot = b.slots(s)
            held = positions.view(b)[page[:settled[s]], slot[:settled[s]]]
            for h in range(Hkv):
                found = held[:, h].tolist()
                assert len(set(found)) == len(found) and (not found or max(found) < seen[s])
                if settled[s] == kv[s]:
                    assert set(range(seen[s] - recent, seen[s])) <= set(found)
        new = [7 * step + 1, 40, 1]
        kv, seen = [t + n for t, n in zip(kv, new)], [t + n for t, n in zip(seen, new)]
    b.ok()


@pytest.mark.parametrize("kv,budget", [(33000, 20000), (40000, 39999), (50001, 7)])
def test_lists_that_no_block_keeps(kv, budget):
    b = _batch([kv], 32, 1, 32, "bf16", "head", seed=1)
    scores = Scores(b, seed=2)
    scores.x.copy_((scores.x * 500).floor())
    _cut(b, scores, [budget], 5)
    b.ok()


@pytest.mark.parametrize("kv,budget,settled", [([9001, 12000], [300, 11990], [300, 8000]), ([70001, 30], [40000, 29], [69000, 11]), ([66000, 131073], [65999, 5000], [0, 66000])])
def test_positions_of_long_lists(kv, budget, settled):
    """Lists that several blocks have, also ones whose keys these do not keep, with positions of their own in front of `settled`; many equal scores."""
    Hkv, recent = 2, 25
    b = _batch(kv, 64, Hkv, 32, "bf16", "head", seed=2)
    scores, positions = Scores(b, seed=5), Scores(b, fill=-5, dtype=torch.int32)
    scores.x.copy_((scores.x * 700).floor())
    seen = [t + 1000 for t in kv]
    for s in range(len(kv)):                            # a cut has left every head with slots in an order of its own
        page, slot = b.slots(s)
        for h in range(Hkv):
            order = torch.randperm(kv[s] + 1000, generator=_gen(h + s), device="cuda")[:settled[s]].to(torch.int32)
            positions.view(b)[page[:settled[s]], slot[:settled[s]], h] = order
    _cut(b, scores, budget, recent, positions, settled, seen)
    b.ok()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset,pad", [(1, 0), (2, 1), (0, 3), (4, 4)])
def test_strides_and_alignment(dtype, offset, pad):
    """Rows that lie on 16 bytes, less, or on their elements only."""
    D, page, Hkv, total = 64, 16, 2, 12
    b = _batch([100, 40], page, Hkv, D, dtype, "head", seed=5)
    total = b.k.shape[0]
    row = D + pad
    flat = [_randn(_gen(i), total * Hkv * page * row + 16, dtype=DT[dtype]) for i in range(2)]
    b.k, b.v = (f[offset:].as_strided((total, Hkv, page, D), (Hkv * page * row, page * row, row, 1), offset) for f in flat)
    b.cache = P.PagedCache(b.k, b.v)
    outside = [f.clone() for f in flat]
    _cut(b, Scores(b, seed=8), [30, 39])
    for f, o, x in zip(flat, outside, (b.k, b.v)):
        o[offset:].as_strided(x.shape, x.stride(), offset).copy_(x)
        assert _same(f, o)                              # nothing between the rows was written
    b.ok()


def test_in_place_lengths_and_refused_sequences():
    """kv_len_out may be kv_len.  A budget below zero or below `recent`, a length beyond the table and one that the scratch was not made for leave the sequence alone and are recorded."""
    b = _batch([100, 90, 80, 200, 70], 16, 2, 64, "bf16", "head", seed=9)
    _cut(b, Scores(b), [50, 90, 30, 100, 69], 10, in_place=True)
    b.ok()
    b = _batch([100, 90, 80, 200, 70, 60], 16, 2, 64, "bf16", "head", seed=9)
    b.kv_len[5] = 10 ** 6
    b.kv[5] = 10 ** 6                                   # (beyond the table: never looked at)
    _cut(b, Scores(b), [50, -1, 5, 100, 9, 5], 10, scratch=_scratch(b, 120), left=(1, 2, 3, 4, 5))
    with pytest.raises(P.EspError):
        b.ok()


def test_a_page_that_there_is_not():
    """It is recorded and touches nothing; the other sequences have their results."""
    b = _batch([64, 64], 16, 2, 64, "bf16", "head", seed=9)
    k0, v0, scores = b.k.clone(), b.v.clone(), Scores(b)
    s0 = scores.x.clone()
    b.table_d[0, 1] = 10 ** 6
    out = torch.empty_like(b.kv_len)
    P.esp_paged_evict(b.cache, b.batch, scores.slots, _i32([20, 20]), out, *_scratch(b))
    with pytest.raises(P.EspError):
        b.ok()
    named = set(b.table[0][[0, 2, 3]].tolist()) | set(b.table[1].tolist())
    for p in set(range(len(k0))) - named:
        assert torch.equal(b.k[p], k0[p]) and torch.equal(b.v[p], v0[p]) and torch.equal(scores.x[p], s0[p])
    b2 = _batch([64, 64], 16, 2, 64, "bf16", "head", seed=9)
    sc2 = Scores(b2)
    P.esp_paged_evict(b2.cache, b2.batch, sc2.slots, _i32([20, 20]), out, *_scratch(b2))
    page, slot = b2.slots(1)
    assert torch.equal(b.view(b.k)[page, slot], b2.view(b2.k)[page, slot])


def test_evict_streams_and_graphs():
    b = _batch([300, 700], 16, 2, 64, "bf16", "head", seed=2)
    scores, scratch = Scores(b), _scratch(b)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _cut(b, scores, [100, 650], 3, stream=side, scratch=scratch)
    # a captured call replayed on other lengths and numbers
    budget, out = _i32([100, 650]), torch.empty_like(b.kv_len)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.esp_paged_evict(b.cache, b.batch, scores.slots, budget, out, *scratch, recent=3)
    b.kv = [200, 690]
    b.kv_len.copy_(_i32(b.kv))
    budget.copy_(_i32([190, 20]))
    scores.x.copy_(torch.rand(scores.x.shape, generator=_gen(77), device="cuda"))
    want = _reference(b, scores.view(b), [190, 20], 3)
    graph.replay()
    torch.cuda.synchronize()
    assert out.tolist() == [190, 20] and _same(b.view(b.k), want[0]) and _same(b.view(b.v), want[1]) and _same(scores.view(b), want[2])


# ================================================================ acceptance
def _accept_reference(b, parents, drafted, chosen, width):
    k, v = b.view(b.k).clone(), b.view(b.v).clone()
    tokens, rows, count, lens = [], [], [], []
    at = b.front
    for s, (n, t) in enumerate(zip(b.n, b.kv)):
        path, row = [], 0 if n and t >= n else None
        while row is not None:
            path.append(row)
            want = chosen[at + row]
            row = next((i for i in range(path[-1] + 1, n) if parents[at + i] == path[-1] and drafted[at + i] == want), None) if want >= 0 else None
        got = [chosen[at + r] if chosen[at + r] >= 0 else -1 for r in path]
        tokens.append(got + [-1] * (width - len(got)))
        rows.append(path + [-1] * (width - len(path)))
        count.append(len(path) - (1 if path and chosen[at + path[-1]] < 0 else 0))
        lens.append(t - n + len(path) if path else t)
        page, slot = b.slots(s)
        new = [[y[page[t - n + r], slot[t - n + r]].clone() for r in path] for y in (k, v)]
        for y, z in zip((k, v), new):
            for i in range(len(path)):
                y[page[t - n + i], slot[t - n + i]] = z[i]
        at += n
    return k, v, tokens, rows, count, lens


def _trees(n, rng, deep):
    """Random trees whose paths are long enough to matter; some rows that hang on nothing, some that name themselves or a later row."""
    parents, drafted, chosen = [], [], []
    for m in n:
        par = [-1] + [int(rng.integers(max(0, i - deep), i)) for i in range(1, m)]
        for i in range(1, m):
            if rng.random() < 0.05:
                par[i] = int(rng.choice([-1, -7, i, i + 1, m + 50]))
        tok = [int(rng.integers(0, 6)) for _ in range(m)]
        cho = [int(rng.integers(0, 6)) for _ in range(m)]
        if m:
            v = int(rng.integers(0, m))
            while v > 0 and 0 <= par[v] < v:               # a path that is right
                cho[par[v]] = tok[v]
                v = par[v]
        parents += par
        drafted += tok
        chosen += cho
    return parents, drafted, chosen


def _accept(b, parents, drafted, chosen, width, rows=True, stream=None):
    i = [_i32([-1] * b.front + x + [3] * (b.tokens - b.front - len(x))) for x in (parents, drafted, chosen)]
    want = _accept_reference(b, *([9] * b.front + x for x in (parents, drafted, chosen)), width)
    out = [torch.full((len(b.n), width), -8, dtype=torch.int32, device="cuda") for _ in range(2)]
    count, lens = torch.full_like(b.kv_len, -8), torch.full_like(b.kv_len, -8)
    P.esp_paged_accept(b.cache, b.batch, *i, out[0], count, lens, rows=out[1] if rows else None, stream=stream)
    torch.cuda.synchronize()
    assert _same(b.view(b.k), want[0]) and _same(b.view(b.v), want[1])
    assert out[0].tolist() == want[2] and count.tolist() == want[4] and lens.tolist() == want[5]
    assert not rows or out[1].tolist() == want[3]


@pytest.mark.parametrize("dtype,Hkv,D,page,order", [("bf16", 2, 128, 16, "head"), ("bf16", 8, 64, 24, "token"), ("fp32", 3, 64, 17, "head"), ("fp32", 1, 32, 1, "token")])
@pytest.mark.parametrize("n,kv", [([1], [1]), ([2], [2]), ([6], [40]), ([128, 1, 0, 68], [300, 9, 33, 68]), ([20] * 50, list(range(20, 70)))])
@pytest.mark.parametrize("deep", [1, 3, 30])
def test_accept(dtype, Hkv, D, page, order, n, kv, deep):
    """Chains, narrow and wide trees; one row, all 128; the first of equal children; rows whose places are sources of others."""
    b = Batch(n, kv, page, Hkv, D, dtype, order, seed=sum(kv), front=2, back=1)
    rng = np.random.default_rng(deep + sum(n))
    for rep in range(3):
        _accept(b, *_trees(n, rng, deep), width=max(n + [1]) + rep, rows=rep != 1)
    b.ok()


def test_accept_a_whole_chain_and_rows_that_chose_nothing():
    b = Batch([128, 5, 4], [200, 30, 4], 16, 2, 64, "bf16", seed=4)
    parents = list(range(-1, 127)) + list(range(-1, 4)) + [-1, 0, 0, 1]
    drafted = list(range(128)) + [9, 8, 7, 6, 5] + [1, 2, 2, 3]
    chosen = list(range(1, 128)) + [-1] + [8, 7, -4, 5, 5] + [2, 3, 3, 1]
    _accept(b, parents, drafted, chosen, 128)
    b.ok()


def test_accept_sequences_that_do_not_hold_together():
    """Padding (kv_len below the rows), a fallen q_start, too many rows: they keep their lengths and pages and are recorded, the others have their results."""
    b = Batch([4, 4, 4], [50, 60, 70], 16, 2, 64, "bf16", seed=4)
    parents, drafted, chosen = [-1, 0, 1, 2] * 3, [0, 1, 2, 3] * 3, [1, 2, 3, 4] * 3
    for what in ("padding", "long", "kv"):
        kv, start = [50, 60, 70], [0, 4, 8, 12]
        if what == "padding":
            kv[1] = 3
        elif what == "long":
            start[1] = 5
        else:
            kv[1] = -1
        out, rows = (torch.empty(3, 4, dtype=torch.int32, device="cuda") for _ in range(2))
        count, lens = torch.empty_like(b.kv_len), torch.empty_like(b.kv_len)
        batch = P.PagedBatch(_i32(start), _i32(kv), b.table_d, 4, b.status)
        k0 = b.k.clone()
        P.esp_paged_accept(b.cache, batch, _i32(parents), _i32(drafted), _i32(chosen), out, count, lens, rows=rows)
        with pytest.raises(P.EspError):
            b.ok()
        b.status.zero_()
        assert torch.equal(b.k, k0)                        # (whole chains stay where they are)
        if what == "long":
            assert count.tolist()[0] == 0 and count.tolist()[2] == 4 and lens.tolist()[0] == 50
        else:
            assert count.tolist() == [4, 0, 4] and lens.tolist() == [50, kv[1], 70] and out[1].tolist() == [-1] * 4 and out[0].tolist() == [1, 2, 3, 4]
