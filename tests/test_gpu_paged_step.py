"""The operators over pages as a server runs them, step after step: append, attention, sampling, acceptance, weights of cached positions, eviction."""
import math

import numpy as np
import pytest
import torch

import paper_2603_17942_b200 as P
from tests.test_gpu_paged import DT, Batch, _gen, _randn
from tests.test_gpu_sample import _check

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Plain:
    """What a head of a sequence remembers: (position, key, value, score) in any order, in 64 bits."""

    def __init__(self):
        self.pos, self.k, self.v, self.score = [], [], [], []


@pytest.mark.parametrize("dtype,D", [("fp32", 64), ("bf16", 64), ("bf16", 128)])
def test_steps_of_a_server(dtype, D):
    """Trees of drafts over cut caches.  The plain side keeps for each head what the head holds, as a set: the device's slots have to hold the same, its attention, tokens and weights have to be the
    formula's.  Attention and weights are as near as their own tests say (a bf16 output 2^-8 of its value, weights of the probabilities 2^-8); scores of two steps differ by more than that is off."""
    B, Hkv, G, page, V, budget, recent, steps = 2, 2, 3, 16, 700, 40, 8, 6
    Hq, prompt = Hkv * G, [50, 23]
    cap = 160
    b = Batch([1] * B, [cap] * B, page, Hkv, D, dtype, seed=2)
    g = _gen(7)
    w_out = _randn(g, Hq * D, V) * 0.6
    scores, positions = (torch.zeros(b.k.shape[:3], dtype=t, device="cuda") for t in (torch.float32, torch.int32))
    s_scores, s_positions = P.PagedSlots(scores), P.PagedSlots(positions)
    settled, seen, kv = _i32([0] * B), list(prompt), list(prompt)
    heads = [[Plain() for _ in range(Hkv)] for _ in range(B)]
    tol = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -18

    def append(n, k, v, length):
        q_start = _i32(np.concatenate([[0], np.cumsum(n)]))
        batch = P.PagedBatch(q_start, _i32(length), b.table_d, max(n), b.status)
        P.esp_paged_append(b.cache, batch, k, v)
        return batch

    def scratch(nb):
        return torch.full((max(nb, 1),), 255, dtype=torch.uint8, device="cuda"), nb

    # the prompts, whose tokens nobody has looked at
    k, v = (_randn(g, sum(prompt), Hkv, D, dtype=DT[dtype]) for _ in range(2))
    append(prompt, k, v, kv)
    at = 0
    for s in range(B):
        for h in range(Hkv):
            for i in range(prompt[s]):
                heads[s][h].pos.append(i)
                heads[s][h].k.append(k[at + i, h].double())
                heads[s][h].v.append(v[at + i, h].double())
                heads[s][h].score.append(0.0)
        at += prompt[s]
    rng = np.random.default_rng(3)
    cuts = accepted = 0
    for step in range(steps):
        n = [int(rng.integers(2, 12)) for _ in range(B)]
        N = sum(n)
        parents = [p for m in n for p in [-1] + [int(rng.integers(0, i)) for i in range(1, m)]]
        q = _randn(g, N, Hq, D, dtype=DT[dtype])
        k, v = (_randn(g, N, Hkv, D, dtype=DT[dtype]) for _ in range(2))
        length = [kv[s] + n[s] for s in range(B)]
        batch = append(n, k, v, length)
        starts = np.concatenate([[0], np.cumsum(n)])
        anc = []
        for s in range(B):
            own = []
            for i in range(n[s]):
                p = parents[starts[s] + i]
                own.append((own[p] if p >= 0 else 0) | (1 << i))
            anc += [[m, 0] for m in own]
        anc_d = torch.tensor(anc, dtype=torch.int64, device="cuda")
        out, lse = torch.empty_like(q), torch.empty(N, Hq, device="cuda")
        P.esp_paged_attention(b.cache, batch, q, out, *scratch(P.esp_paged_attention_scratch_bytes(Hq, D)), anc=anc_d, lse=lse)
        # the plain attention of every row over what its head holds and its ancestors
        for s in range(B):
            for i in range(n[s]):
                row = starts[s] + i
                up = [starts[s] + j for j in range(n[s]) if (anc[row][0] >> j) & 1]
                for e in range(Hq):
                    held = heads[s][e // G]
                    ks, vs = torch.stack(held.k + [k[j, e // G].double() for j in up]), torch.stack(held.v + [v[j, e // G].double() for j in up])
                    x = ks @ q[row, e].double() / math.sqrt(D)
                    w = torch.softmax(x, 0)
                    want = w @ vs
                    assert abs(float(torch.logsumexp(x, 0)) - float(lse[row, e])) < 2.0 ** -15
                    assert (out[row, e].double() - want).norm() <= 2 * tol * want.norm() + 2.0 ** -20
        logits = out.float().reshape(N, -1) @ w_out
        u = torch.rand(N, generator=g, device="cuda")
        tokens, logprob = torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, device="cuda")
        settings = dict(temperature=torch.full((N,), 0.8, device="cuda"), top_k=_i32([30] * N), top_p=torch.full((N,), 0.9, device="cuda"))
        P.esp_sample(logits, u, tokens, *scratch(P.esp_sample_scratch_bytes(N, V)), logprob=logprob, **settings)
        _check(logits, u.cpu().numpy(), tokens, logprob, temperature=np.float32(0.8), top_k=30, top_p=np.float32(0.9))
        # drafts of which some are what the model says
        chosen = tokens.tolist()
        drafted = [-1 if p < 0 else (chosen[starts[np.searchsorted(starts, r, side="right") - 1] + p] if rng.random() < 0.6 else int(rng.integers(V))) for r, p in enumerate(parents)]
        tok, rows = (torch.empty(B, max(n), dtype=torch.int32, device="cuda") for _ in range(2))
        n_out, kv_out = _i32([0] * B), _i32([0] * B)
        P.esp_paged_accept(b.cache, batch, _i32(parents), _i32(drafted), tokens, tok, n_out, kv_out, rows=rows)
        paths = []
        for s in range(B):
            path, r = [], 0
            while r is not None:
                path.append(r)
                r = next((i for i in range(n[s]) if parents[starts[s] + i] == path[-1] and drafted[starts[s] + i] == chosen[starts[s] + path[-1]]), None)
            paths.append(path)
            assert rows[s, :len(path)].tolist() == path and int(n_out[s]) == len(path) and int(kv_out[s]) == kv[s] + len(path)
            assert tok[s, :len(path)].tolist() == [chosen[starts[s] + r] for r in path]
        accepted += sum(len(p) - 1 for p in paths)
        # what the accepted rows looked at: their lse under the tree's mask is theirs over the compacted cache
        pick = torch.tensor([starts[s] + r for s in range(B) for r in paths[s]], device="cuda")
        m = [len(p) for p in paths]
        kv = kv_out.tolist()
        batch = P.PagedBatch(_i32(np.concatenate([[0], np.cumsum(m)])), kv_out, b.table_d, max(m), b.status)
        P.esp_paged_key_weights(b.cache, batch, q[pick], lse[pick].contiguous(), s_scores, *scratch(P.esp_paged_key_weights_scratch_bytes(sum(m), Hq, D)), keep=0.5)
        for s in range(B):
            for h in range(Hkv):
                held = heads[s][h]
                old = len(held.pos)
                held.score = [0.5 * x for x in held.score] + [0.0] * m[s]
                for i, r in enumerate(paths[s]):
                    held.pos.append(seen[s] + i)
                    held.k.append(k[starts[s] + r, h].double())
                    held.v.append(v[starts[s] + r, h].double())
                for i, r in enumerate(paths[s]):
                    for e in range(h * G, (h + 1) * G):
                        x = torch.stack(held.k[:old + i + 1]) @ q[starts[s] + r, e].double() / math.sqrt(D)
                        for j, w in enumerate((x - lse[starts[s] + r, e].double()).exp().tolist()):
                            held.score[j] += w
            seen[s] += m[s]
        # the cut, on the scores as the device has them
        P.esp_paged_evict(b.cache, batch, s_scores, _i32([budget] * B), kv_out, *scratch(P.esp_paged_evict_scratch_bytes(B, Hkv, cap)), recent=recent, positions=s_positions, settled=settled,
                          seen=_i32(seen))
        before, kv = kv, kv_out.tolist()
        for s in range(B):
            assert kv[s] == min(before[s], budget)
            cuts += before[s] > budget
            page_, slot = (x[:kv[s]] for x in b.slots(s))
            for h in range(Hkv):
                held = heads[s][h]
                here = positions[page_, h, slot].tolist() if int(settled[s]) else list(range(kv[s]))
                stay = dict(zip(here, range(kv[s])))
                assert len(stay) == kv[s] and set(range(max(0, seen[s] - recent), seen[s])) <= set(stay)
                gone = [x for p, x in zip(held.pos, held.score) if p not in stay]
                kept = {p: i for i, p in enumerate(held.pos) if p in stay}
                # the lowest kept score of the older ones is not below the highest dropped one (2^-12: what a weight is off by here at most)
                old = [held.score[i] for p, i in kept.items() if p < seen[s] - recent]
                assert not gone or not old or min(old) >= max(gone) * (1 - 2.0 ** -12) - 1e-9
                order = [kept[p] for p in here]
                got = scores[page_, h, slot].double().cpu().numpy()
                assert np.allclose(got, [held.score[i] for i in order], rtol=2.0 ** -12, atol=1e-7)
                assert torch.equal(b.k[page_, h, slot].double(), torch.stack([held.k[i] for i in order])) and torch.equal(b.v[page_, h, slot].double(), torch.stack([held.v[i] for i in order]))
                held.pos, held.k, held.v, held.score = here, [held.k[i] for i in order], [held.v[i] for i in order], [held.score[i] for i in order]
        b.ok()
    assert cuts >= steps and accepted > 0
