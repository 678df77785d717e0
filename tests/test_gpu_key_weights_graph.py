"""The attention that cached positions receive, read by what comes next in the same captured graph."""
import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_gpu_key_weights import DT, Batch, Scores, _check, _gen, _lse, _randn, _scratch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,Hkv,D,n,kv", [("bf16", 8, 2, 128, [32, 7, 30, 1], [4000, 2100, 5000, 3000]), ("fp32", 8, 2, 64, [8, 3, 5], [3000, 2100, 900]), ("bf16", 4, 2, 32, [9, 16], [3000, 70]),
                                                 ("bf16", 8, 2, 128, [68, 40], [4000, 2100])])
def test_scores_copied_behind_the_call(dtype, Hq, Hkv, D, n, kv):
    """max_new above the tokens of every sequence, so that a join is launched although (but for the last set) no chunk has two owners: a copy behind it in the graph has all scores."""
    b = Batch(n, kv, 16, Hkv, D, dtype, seed=7)
    q = _randn(_gen(1), b.tokens, Hq, D, dtype=DT[dtype])
    lse = _lse(b, q)
    batch = P.PagedBatch(b.q_start, b.kv_len, b.table_d, 68, b.status)
    scores, scratch = Scores(b), _scratch(b, q)
    out, large, start = torch.empty_like(scores.flat), torch.empty(1 << 26, device="cuda"), scores.flat.clone()
    P.esp_paged_key_weights(b.cache, batch, q, lse, scores.slots, *scratch, keep=0.0)
    _check(b, q, lse, Scores(b).x, scores, 0.0)
    eager = scores.flat.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        scores.flat.copy_(start)
        P.esp_paged_key_weights(b.cache, batch, q, lse, scores.slots, *scratch, keep=0.0)
        out.copy_(scores.flat)
    for i in range(60):
        if i % 10 == 0:
            large.fill_(i)                # (the keys are out of the cache: the weights' kernel takes longer)
        out.fill_(-3.0)
        graph.replay()
        assert torch.equal(out, eager), i
    b.ok()
