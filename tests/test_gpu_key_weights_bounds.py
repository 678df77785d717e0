"""The attention that cached positions receive, with bounds far above what the call has."""
import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_gpu_key_weights import DT, Batch, Scores, _check, _gen, _lse, _randn, _scratch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page", [("bf16", 8, 2, 128, 17), ("bf16", 14, 2, 64, 9), ("bf16", 8, 2, 128, 16), ("fp32", 8, 2, 64, 16), ("bf16", 8, 2, 32, 16)])
@pytest.mark.parametrize("n,kv", [([60], [300]), ([5, 130, 1], [600, 400, 9])])
@pytest.mark.parametrize("max_new", [2 ** 31 - 1, 2 ** 30 + 1, 2 ** 30])
@pytest.mark.parametrize("last", [0, 2 ** 31 - 1, 3])
def test_max_new_is_a_bound(dtype, Hq, Hkv, D, page, n, kv, max_new, last):
    """2^31 - 1 is one too; so it is for the observed tokens."""
    b = Batch(n, kv, page, Hkv, D, dtype, seed=D + page)
    q = _randn(_gen(3), b.tokens, Hq, D, dtype=DT[dtype])
    lse, scores = _lse(b, q), Scores(b)
    before = scores.x.clone()
    P.esp_paged_key_weights(b.cache, P.PagedBatch(b.q_start, b.kv_len, b.table_d, max_new, b.status), q, lse, scores.slots, *_scratch(b, q), last=last, keep=0.5)
    _check(b, q, lse, before, scores, 0.5, last=last)
    b.ok()
