"""The operators over a paged cache at the edges of what their header promises.  Tolerances as in test_gpu_paged.py."""
import math

import pytest
import torch

from tests.test_gpu_paged import DT, NAN, Batch, _attention, _check_attention, _gen, _randn

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
