"""Cutting caches whose tables have room for far more positions than the sequences hold, and calls that mix short lists with long ones: equal bit by bit to plain loops."""
import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_gpu_key_weights import Scores
from tests.test_gpu_paged_evict import _batch, _cut, _scratch

pytestmark = pytest.mark.gpu


def _widen(b, positions):
    """The batch's table with rows for that many positions; entries that nobody needs name no page."""
    table = torch.full((len(b.kv), -(-positions // b.page)), -1, dtype=torch.int32, device="cuda")
    table[:, :b.table_d.shape[1]] = b.table_d
    b.batch = P.PagedBatch(b.q_start, b.kv_len, table, 1, b.status)


@pytest.mark.parametrize("room", [8192, 8208, 33000, 70000, 1 << 20])
@pytest.mark.parametrize("held", [None, 8192, 65536, 1 << 18])
@pytest.mark.parametrize("kv,budget,Hkv", [([300, 77, 40], [200, 77, 1], 2), ([650] * 40, list(range(610, 650)), 8)])
def test_tables_with_room(room, held, kv, budget, Hkv):
    """Scratch for what the sequences hold and for much longer lists; few lists and more than there are blocks at a time."""
    b = _batch(kv, 16, Hkv, 64, "bf16", "head", seed=room)
    _widen(b, room)
    scores, positions = Scores(b, seed=3), Scores(b, fill=-5, dtype=torch.int32)
    scores.x.copy_((scores.x * 200).floor())
    settled = [t // 2 for t in kv]
    for s, t in enumerate(kv):
        page, slot = b.slots(s)
        positions.view(b)[page[:settled[s]], slot[:settled[s]]] = torch.arange(settled[s], dtype=torch.int32, device="cuda")[:, None]
    _cut(b, scores, budget, 1, positions, settled, [t + 9 for t in kv], scratch=_scratch(b, held))
    b.ok()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("long", [8193, 20000, 70001])
def test_short_lists_beside_long_ones(dtype, long):
    """Lists of one block and of a cluster in one call, at the border of what a block keeps, below their budgets and empty."""
    kv = [long, 8192, 8191, 5, 0, 300, 8193] + [40 + s for s in range(60)]
    budget = [long // 3, 8191, 100, 4, 0, 400, 4000] + [30 + s % 11 for s in range(60)]
    b = _batch(kv, 32, 3, 32, dtype, "token", seed=long)
    scores = Scores(b, seed=2)
    scores.x.copy_((scores.x * 3000).floor())
    _cut(b, scores, budget, 2)
    b.ok()
