"""The operators over a paged cache at the edges of what their header promises.  Tolerances as in test_gpu_paged.py."""
import math

import numpy as np
import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_gpu_paged import DT, NAN, Batch, _attention, _check_attention, _check_norm_rope, _gen, _layer, _randn, _rope_table

pytestmark = pytest.mark.gpu


# ================================================================ infinite values that a single token sees
@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 16, 2, 128), ("bf16", 16, 1, 128), ("bf16", 9, 1, 128), ("bf16", 4, 1, 64), ("bf16", 16, 2, 64),
                                            ("bf16", 32, 2, 64), ("bf16", 8, 2, 32), ("fp32", 8, 2, 64)])
@pytest.mark.parametrize("kv", [[1], [2, 33, 1], [400, 97, 31], [5000], [700] * 150])
@pytest.mark.parametrize("window", [0, 90])
def test_an_infinite_value_that_a_single_token_sees_stays_infinite(dtype, Hq, Hkv, D, kv, window):
    """Weights of exactly 1 (one visible key), ordinary ones, tiles of one worker and tiles that many share, the first and last positions of a stage and of the window: an
    infinite value makes its dimension infinite, values of both signs and values that are no numbers make it undefined, all else keeps its bits."""
    b = Batch([1] * len(kv), kv, 16, Hkv, D, dtype, seed=len(kv) + D)
    q = _randn(_gen(21), len(kv), Hq, D, dtype=DT[dtype])
    clean, l0 = _attention(b, q, window=window)
    _check_attention(b, q, clean, l0, window=window)
    want = clean.clone()
    for s, t in enumerate(kv):
        pg, sl = b.slots(s)
        spoil = [(t - 1, 3, math.inf), (t - 1, 8, NAN), (0, 9, -math.inf), (0, 17, math.inf), (t - 1, 17, -math.inf), (t // 2, 21, math.inf), (t // 2, 30, -math.inf),
                 (max(0, t - 90), 6, math.inf), (max(0, t - 91), 7, math.inf), (min(31, t - 1), 12, -math.inf), (min(32, t - 1), 13, math.inf)]
        for p, d, x in spoil:
            b.view(b.v)[pg[p], sl[p], :, d] = x
        # what each dimension of v sums up to where it is not finite
        lo = max(0, t - window) if window else 0
        v = b.read(b.v, s)[lo:].double()                                      # [seen, Hkv, D]
        odd = torch.where(v.isfinite(), 0.0, v).sum(0).repeat_interleave(Hq // Hkv, 0)
        want[s] = torch.where(odd == 0, want[s].double(), odd).to(want.dtype)
        touched = torch.zeros(D, dtype=torch.bool, device="cuda")
        touched[[d for p, d, x in spoil if p >= lo]] = True
        assert torch.equal((odd != 0), touched.expand(Hq, D))
    got, l1 = _attention(b, q, window=window)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[~want.isnan()], want[~want.isnan()])
    assert torch.equal(l0, l1)
    b.ok()


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 14, 2, 64), ("bf16", 8, 2, 32), ("fp32", 8, 2, 64)])
def test_an_infinite_value_that_every_token_sees_stays_infinite(dtype, Hq, Hkv, D):
    """Blocks of several tokens: chunks that every row sees as a whole, tiles that many share, chunks that go through both sets of scores in turn."""
    n, kv = [70, 5, 9], [1000, 300, 20000]
    b = Batch(n, kv, 16, Hkv, D, dtype, seed=D)
    q = _randn(_gen(23), b.tokens, Hq, D, dtype=DT[dtype])
    want, _ = _attention(b, q)
    at = 0
    for s in range(3):
        pg, sl = b.slots(s)
        for p, d, x in [(0, 1, math.inf), (127, 2, -math.inf), (128, 30, NAN), (200, 19, math.inf), (201, 19, -math.inf), (kv[s] - n[s], 21, math.inf), (kv[s] // 2, 7, math.inf)]:
            b.view(b.v)[pg[p], sl[p], :, d] = x
            want[at:at + n[s], :, d] = want[at:at + n[s], :, d] + x if d == 19 and x < 0 else x
        at += n[s]
    got, _ = _attention(b, q)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[~want.isnan()], want[~want.isnan()])
    b.ok()


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 64), ("bf16", 32, 2, 64), ("bf16", 8, 2, 128), ("bf16", 16, 1, 128), ("bf16", 8, 2, 32), ("fp32", 8, 2, 64)])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("kv", [[300], [3000], [200] * 60])
def test_an_infinite_value_of_a_small_weight(dtype, Hq, Hkv, D, n, kv):
    """Keys whose logits are 90 below the others' in powers of two (the header's bound is 100): queries are 4, their keys -c with 4 c D scale log2(e) = 90 up to the rounding of
    c, all other keys zero; before, between and behind the others."""
    b = Batch([n] * len(kv), kv, 16, Hkv, D, dtype, seed=D, fill=0.0)
    c = 90 / (4 * D ** 0.5 * math.log2(math.e))
    want = torch.zeros(b.tokens, Hq, D, dtype=DT[dtype], device="cuda")
    for s, t in enumerate(kv):
        pg, sl = b.slots(s)
        for d, p in enumerate((0, 1, 130, t // 2, t - n)):            # (every token sees them)
            b.view(b.k)[pg[p], sl[p]] = -c
            b.view(b.v)[pg[p], sl[p], :, d] = math.inf if d % 2 else -math.inf
            want[s * n:(s + 1) * n, :, d] = math.inf if d % 2 else -math.inf
        if n == 1:                                                     # (t - n is the token itself: left finite)
            b.view(b.k)[pg[t - 1], sl[t - 1]] = 0.0
            b.view(b.v)[pg[t - 1], sl[t - 1]] = 0.0
            want[s, :, 4] = 0.0
    q = torch.full((b.tokens, Hq, D), 4.0, dtype=DT[dtype], device="cuda")
    out, _ = _attention(b, q)
    assert torch.equal(out, want)
    b.ok()


# ================================================================ page tables with holes
@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 16, 1, 64), ("fp32", 4, 2, 64), ("bf16", 3, 1, 32)])
@pytest.mark.parametrize("page", [16, 64, 24, 5])
@pytest.mark.parametrize("n,kv", [([1, 1, 1], [400, 97, 1031]), ([50, 1, 300], [400, 97, 1031])])
@pytest.mark.parametrize("window", [1, 90, 130])
def test_pages_behind_every_window_need_no_entry(dtype, Hq, Hkv, D, page, n, kv, window):
    """A server that gives the pages behind the window back leaves no page number there: positions that no token sees are not looked up, and nothing is recorded."""
    b = Batch(n, kv, page, Hkv, D, dtype, seed=page + window)
    q = _randn(_gen(22), b.tokens, Hq, D, dtype=DT[dtype])
    full, l0 = _attention(b, q, window=window)
    _check_attention(b, q, full, l0, window=window)
    for s in range(len(n)):
        first = max(0, kv[s] - n[s] - window + 1)                 # what the sequence's first token sees first
        b.table_d[s, :first // page] = -1
        if first // page > 1:
            b.table_d[s, 1] = 2 ** 31 - 1
    assert bool((b.table_d[0] == -1).any())
    got, l1 = _attention(b, q, window=window)
    assert torch.equal(got, full) and torch.equal(l0, l1)
    b.ok()


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("stride", [1 << 39, 1 << 40])
def test_page_strides_that_a_tensor_map_cannot_hold(n, stride):
    """Pages 2^40 bytes and more apart, of which the table names the first alone: such a cache goes the way of those that no tensor map fits."""
    b = Batch([n, 1], [60, 48], 64, 2, 128, "bf16", seed=3)
    x = _randn(_gen(28), b.tokens, 12, 128, dtype=torch.bfloat16)
    b.n, b.kv = [n, 0], [60, 0]
    b.table[0, 0], b.unused = 0, None
    b.table_d[0, 0] = 0
    b.q_start.copy_(torch.tensor([0, n, n], dtype=torch.int32))
    b.kv_len.copy_(torch.tensor([60, 0], dtype=torch.int32))
    P.esp_paged_append(b.cache, b.batch, x[:, 8:10], x[:, 10:])
    want, l0 = _attention(b, x[:, :8])
    b.cache.c.page_stride = stride
    P.esp_paged_append(b.cache, b.batch, x[:, 8:10], x[:, 10:])
    got, l1 = _attention(b, x[:, :8])
    _check_attention(b, x[:, :8], want, l0)
    _check_attention(b, x[:, :8], got, l1)


# ================================================================ descriptions that contradict each other
class One:
    """Sequence s of a batch on its own, for _check_attention."""

    def __init__(self, b, s, start, n):
        self.n, self.kv, self.front, self.k, self.v, self.order = [n], [b.kv[s]], start, b.k, b.v, b.order
        self.read = lambda x, _: b.read(x, s)
        self.ok = lambda: None


def _check_served(b, q, out, lse, starts, served):
    """Every served sequence has its results, all other rows of out and lse are as they were."""
    mine = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for s in served:
        mine[starts[s]:starts[s + 1]] = True
    assert bool((out[~mine] == 7.0).all()) and bool((lse[~mine] == 7.0).all())
    for s in served:
        keep = torch.full_like(out, 7.0)
        keep[starts[s]:starts[s + 1]] = out[starts[s]:starts[s + 1]]
        _check_attention(One(b, s, starts[s], starts[s + 1] - starts[s]), q, keep, lse)


def _check_appended(b, k, v, k0, v0, starts, served):
    """The slots of the served sequences hold their tokens, every other one its bits."""
    for s in served:
        n = starts[s + 1] - starts[s]
        pg, sl = (x[b.kv[s] - n:] for x in b.slots(s))
        b.view(k0)[pg, sl], b.view(v0)[pg, sl] = k[starts[s]:starts[s + 1]], v[starts[s]:starts[s + 1]]
    assert torch.equal(b.k, k0) and torch.equal(b.v, v0)


def _recorded(b):
    with pytest.raises(P.EspError) as e:
        P.esp_paged_status(b.batch)
    assert e.value.code == -5
    b.status.zero_()


OVERLAPS = {
    "later sequence inside an earlier one": ([0, 100, 50, 120, 130], [0, 3]),
    "starts before it fell": ([60, 20, 80, 100, 130], [1, 2, 3]),
    "one inside two": ([0, 40, 90, 30, 70, 130], [0, 1]),
    "falls behind the last": ([0, 60, 130, 20], [0, 1]),
    "single tokens": (list(range(100)) + list(range(60, 130)), list(range(99)) + list(range(139, 169))),
    "very many": (list(range(400)) + list(range(300, 500)), list(range(399)) + list(range(499, 599))),
}


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 8, 2, 128), ("fp32", 4, 2, 64)])
@pytest.mark.parametrize("what", list(OVERLAPS))
@pytest.mark.parametrize("spare", [0, 6])               # a bound above 1: the kernel of several tokens
def test_no_token_has_two_owners(dtype, Hq, Hkv, D, what, spare):
    """Where q_start falls, a later sequence may claim tokens that an earlier one has: the earlier one has them, the later one is left out as a whole, in the attention and in
    the append; who does not overlap is served; the same call gives the same bits."""
    starts, served = OVERLAPS[what]
    B, tokens = len(starts) - 1, max(starts) + 3
    most = max(starts[s + 1] - starts[s] for s in range(B))
    kv = [130 + 7 * s % 50 for s in range(B)]
    b = Batch([1] * B, kv, 16, Hkv, D, dtype, seed=B)
    b.q_start.copy_(torch.tensor(starts, dtype=torch.int32))
    b.batch = P.PagedBatch(b.q_start, b.kv_len, b.table_d, most + spare, b.status)
    x = _randn(_gen(24), tokens, Hq + 2 * Hkv, D, dtype=DT[dtype])
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    k0, v0 = b.k.clone(), b.v.clone()
    P.esp_paged_append(b.cache, b.batch, k, v)
    _recorded(b)
    _check_appended(b, k, v, k0, v0, starts, served)
    out, lse = _attention(b, q)
    _recorded(b)
    _check_served(b, q, out, lse, starts, served)
    again, _ = _attention(b, q)
    _recorded(b)
    assert torch.equal(out, again)


@pytest.mark.parametrize("n", [1, 50])
def test_who_holds_together_has_its_results(n):
    """Beside a sequence whose numbers contradict each other, or whose table names a page that there is not, the others have the results of their own keys and values, and
    the append writes their slots alone."""
    x = _randn(_gen(30), 3 * n, 12, 128, dtype=torch.bfloat16)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    whole = [0, n, 2 * n, 3 * n]
    changes = [
        (lambda b: b.kv_len[1:2].fill_(b.table.shape[1] * 16 + 1), whole, [0, 2]),
        (lambda b: b.kv_len[1:2].fill_(-1), whole, [0, 2]),
        (lambda b: b.kv_len[0:1].fill_(2 ** 31 - 1), whole, [1, 2]),
        (lambda b: b.q_start[3:].fill_(3 * n + 1), whole[:3] + [3 * n + 1], [0, 1]),
        (lambda b: b.q_start[1:2].fill_(2 * n + 1), [0, 2 * n + 1, 2 * n, 3 * n], [2]),       # the first has too many tokens, the second falls
        (lambda b: b.q_start[:1].fill_(-1), [-1, n, 2 * n, 3 * n], [1, 2]),
    ]
    for change, starts, served in changes:
        b = Batch([n, n, n], [100, 200, 300], 16, 2, 128, "bf16", seed=2)
        change(b)
        k0, v0 = b.k.clone(), b.v.clone()
        P.esp_paged_append(b.cache, b.batch, k, v)
        _recorded(b)
        _check_appended(b, k, v, k0, v0, starts, served)
        out, lse = _attention(b, q)
        _recorded(b)
        _check_served(b, q, out, lse, starts, served)
    for page in (-1, b.k.shape[0], 2 ** 31 - 1):                          # the page of the second sequence's positions 192 .. 199
        b = Batch([n, n, n], [100, 200, 300], 16, 2, 128, "bf16", seed=2)
        lost = int(b.table[1, 12])
        b.table_d[1, 12] = page
        k0, v0 = b.k.clone(), b.v.clone()
        P.esp_paged_append(b.cache, b.batch, k, v)
        _recorded(b)
        pages = b.k[lost].clone(), b.v[lost].clone()
        assert torch.equal(pages[0], k0[lost]) and torch.equal(pages[1], v0[lost])
        if n == 1:                                                        # (the only new token of the second sequence has no slot)
            _check_appended(b, k, v, k0, v0, whole, [0, 2])
        out, lse = _attention(b, q)
        _recorded(b)
        out[n:2 * n], lse[n:2 * n] = 7.0, 7.0                             # no promise about its own rows
        _check_served(b, q, out, lse, whole, [0, 2])


# ================================================================ every position, one by one
@pytest.mark.parametrize("Hq,Hkv,D,page,n,kv", [(16, 8, 128, 64, [16, 9, 1, 3, 30], [32100, 29999, 16000, 1, 30]), (16, 8, 64, 16, [4] * 6, [30000 - 77 * i for i in range(6)]),
                                               (8, 2, 128, 16, [130, 70], [5000, 3333]), (8, 2, 64, 24, [1] * 5, [9000, 31, 4099, 1, 20000])])
def test_every_position_has_its_own_share(Hq, Hkv, D, page, n, kv):
    """Queries of zero weigh the t visible keys alike.  Values are 1 in dim p - first for the D positions from `first` on and zero elsewhere, one call for each `first`: an output is
    1 / t for each of those positions that is seen, 0 for the others, so that a position lost or counted twice is an error of the whole value.  Tiles of few pairs
    whose chunks go through both sets of scores in turn, tiles of two subtiles, single tokens.  Roundings: weights and 1 are exact, the output is rounded once."""
    b = Batch(n, kv, page, Hkv, D, "bf16", seed=3, fill=0.0)
    q = torch.zeros(b.tokens, Hq, D, device="cuda", dtype=torch.bfloat16)
    seen = torch.cat([torch.arange(t - m + 1, t + 1) for m, t in zip(n, kv)]).clamp(min=0).cuda()     # t of every token; 0: padding
    eye = torch.eye(D, device="cuda", dtype=torch.bfloat16)[:, None].expand(-1, Hkv, -1)
    slots = [b.slots(s) for s in range(len(n))]
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for first in range(0, max(kv), D):
        for (pg, sl), t in zip(slots, kv):
            last = min(first + D, t)
            if first < last:
                b.view(b.v)[pg[first:last], sl[first:last]] = eye[:last - first]
        out, _ = _attention(b, q, lse=False)
        want = torch.where(first + torch.arange(D, device="cuda") < seen[:, None], 1.0 / seen.clamp(min=1)[:, None].double(), 0.0)[:, None]
        wrong += ((out.double() - want).abs() > 2.0 ** -8 * 1.01 * want).sum()
        for (pg, sl), t in zip(slots, kv):
            last = min(first + D, t)
            if first < last:
                b.view(b.v)[pg[first:last], sl[first:last]] = 0.0
    assert int(wrong) == 0
    b.ok()


# ================================================================ streams
def test_calls_without_a_stream_are_ordered_with_their_tensors():
    """Under torch.cuda.stream() a call that names no stream runs behind the work that makes its inputs and before the work that reads its outputs."""
    Hq, Hkv, D = 8, 2, 128
    b = Batch([1, 40], [300, 200], 16, Hkv, D, "bf16", seed=1)
    cfg = P.rope_cfg(D)
    good = _randn(_gen(25), b.tokens, Hq + 2 * Hkv, D, dtype=torch.bfloat16)
    x = torch.zeros_like(good)
    pos = torch.arange(b.tokens, dtype=torch.int32, device="cuda")
    k_out = torch.zeros(b.tokens, Hkv, D, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        table = _rope_table(cfg)
        torch.cuda._sleep(100_000_000)                    # about 50 ms
        x.copy_(good)
        P.esp_qk_norm_rope(None, x[:, Hq:Hq + Hkv], None, k_out, cfg, table, pos)
        q, out = _layer(b, x, cfg, table, [None, None])
        kept = q.clone(), out.clone(), k_out.clone()
        b.ok()                                            # waits for this stream
        done = side.query()
    assert done
    torch.cuda.synchronize()
    _check_attention(b, kept[0], kept[1], None)
    _check_norm_rope(kept[2], good[:, Hq:Hq + Hkv], pos.cpu().numpy(), cfg, None, 0, "bf16")


def test_captured_without_naming_the_stream():
    Hq, Hkv, D = 8, 2, 64
    b = Batch([1, 1], [300, 200], 16, Hkv, D, "bf16", seed=1)
    cfg = P.rope_cfg(D)
    table = _rope_table(cfg)
    x = _randn(_gen(26), b.tokens, Hq + 2 * Hkv, D, dtype=torch.bfloat16)
    q, out = torch.empty(b.tokens, Hq, D, device="cuda", dtype=torch.bfloat16), torch.empty(b.tokens, Hq, D, device="cuda", dtype=torch.bfloat16)
    nb = P.esp_paged_attention_scratch_bytes(Hq, D)
    scratch = torch.empty(nb, dtype=torch.uint8, device="cuda"), nb
    _layer(b, x, cfg, table, [None, None], q_out=q, out=out, scratch=scratch)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _layer(b, x, cfg, table, [None, None], q_out=q, out=out, scratch=scratch)
    x.copy_(_randn(_gen(27), *x.shape))
    out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    _check_attention(b, q, out, None)

# ================================================================ the angle of a position
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D", [64, 36])                   # wide accesses, and one element at a time
def test_the_angle_is_off_by_its_rounding_to_fp32_at_most(D, interleaved):
    """Pairs (1, 0) come out as (cos, sin): off by the angle's rounding (2^-26 of a turn), the table's (2^-31), and two roundings of the sine; the reference's frequency
    in fp64 adds position * 2^-53 rad."""
    cfg = P.rope_cfg(D, 500000.0, interleaved=interleaved)
    pos = torch.randint(-2 ** 24, 2 ** 24, (4000,), generator=_gen(29), device="cuda", dtype=torch.int32)
    x = torch.zeros(4000, 1, D, device="cuda")
    first = torch.arange(0, D, 2) if interleaved else torch.arange(D // 2)
    second = first + (1 if interleaved else D // 2)
    x[..., first] = 1.0
    out = torch.empty_like(x)
    P.esp_qk_norm_rope(x, None, out, None, cfg, _rope_table(cfg), pos)
    p = pos.cpu().numpy().astype(np.longdouble)
    angle = p[:, None] * P.esp_rope_frequencies(cfg).astype(np.longdouble)
    tol = 2 * np.pi * (2.0 ** -26 + 2.0 ** -31) + 2 * 2.0 ** -24 + np.abs(p.astype(np.float64))[:, None] * 2.0 ** -53
    got = out[:, 0].double().cpu().numpy()
    for at, f in ((first, np.cos), (second, np.sin)):
        assert bool((np.abs(got[:, at.numpy()] - f(angle).astype(np.float64)) <= tol).all())
