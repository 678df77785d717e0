"""The attention that cached positions receive, in calls with sequences that are padded far: kv_len well below the number of new tokens, down to none at all."""
import pytest
import torch

from tests.test_gpu_key_weights import DT, Batch, _gen, _randn, _run

pytestmark = pytest.mark.gpu

# (tokens, positions): alone and between two ordinary sequences
PADDED = [([2000], [0]), ([2000], [1]), ([807], [234]), ([543], [0]), ([205], [65]), ([200], [10]), ([3000], [2000]), ([600, 5], [10, 300]), ([600, 5], [0, 300]), ([200, 900], [40, 400]),
          ([5, 2000, 70], [300, 0, 90]), ([70, 2000, 3], [300, 1, 90]), ([130, 807, 7], [300, 234, 90]), ([40, 205, 9], [50, 65, 700]), ([40, 200, 9], [50, 10, 700])]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page", [("bf16", 8, 2, 128, 16), ("bf16", 14, 2, 64, 24), ("bf16", 8, 2, 128, 17), ("fp32", 8, 2, 64, 16), ("bf16", 4, 2, 32, 16)])
@pytest.mark.parametrize("n,kv", PADDED)
@pytest.mark.parametrize("window,last", [(0, 0), (0, 300), (50, 0)])
def test_far_padding(dtype, Hq, Hkv, D, page, n, kv, window, last):
    """Every sequence of the call has its scores and nothing is recorded, whatever one of them is padded by."""
    b = Batch(n, kv, page, Hkv, D, dtype, seed=sum(n) + D, front=1, back=2)
    q = _randn(_gen(3), b.tokens, Hq, D, dtype=DT[dtype], scale=2.0)
    _run(b, q, 0.75, window=window, last=last)


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page", [("bf16", 8, 2, 128, 16), ("bf16", 8, 2, 64, 9), ("fp32", 8, 2, 32, 16)])
@pytest.mark.parametrize("count", [31, 45, 70])
def test_many_sequences_of_several_tiles(dtype, Hq, Hkv, D, page, count):
    """More sequences than a warp has lanes, of several tiles each; a third of them padded, some far."""
    g = torch.Generator().manual_seed(count)
    n = torch.randint(1, 420, (count,), generator=g).tolist()
    kv = [max(0, m + (int(torch.randint(0, 500, (1,), generator=g)) if s % 3 else -int(torch.randint(0, 420, (1,), generator=g)))) for s, m in enumerate(n)]
    n[4], kv[4], n[9] = 700, 3, 0
    b = Batch(n, kv, page, Hkv, D, dtype, seed=count, front=2)
    q = _randn(_gen(5), b.tokens, Hq, D, dtype=DT[dtype])
    _run(b, q, 0.5)
    _run(b, q, 0.0, last=100)
