"""Sampling from large vocabularies whose logits hardly differ: most of a row's weight in one bin of a histogram, its front's end far behind that."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import _call, _check

pytestmark = pytest.mark.gpu


def _flat(vocab, dtype, seed):
    """Nine tenths of the logits just below 0.04, the rest spread over lower ones, a few above."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = 0.0396 + 0.0003 * torch.rand(vocab, generator=g, device="cuda")
    low = torch.rand(vocab, generator=g, device="cuda") < 0.1
    x[low] = -8 * torch.rand(int(low.sum()), generator=g, device="cuda")
    x[torch.randint(0, vocab, (50,), generator=g, device="cuda")] = 0.7
    return x.to(dtype)[None]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [2 ** 21, 2 ** 20 + 5, 2 ** 21 - 3])
def test_fronts_behind_a_full_bin(dtype, vocab):
    """Rows one by one and more of them than there are clusters of eight, where a block has twice the logits."""
    x = _flat(vocab, dtype, vocab)
    rows = 190
    p, u = np.linspace(0.9, 0.99995, rows).astype(np.float32), np.random.default_rng(1).random(rows).astype(np.float32)
    tokens, lp = _call(x.expand(rows, vocab), u, top_p=p)
    for i in (0, 60, 120, 150, 189):
        _check(x, u[i:i + 1], tokens[i:i + 1], lp[i:i + 1], top_p=p[i:i + 1])
        one, _ = _call(x, u[i:i + 1], top_p=p[i:i + 1])
        assert one[0] == tokens[i]
