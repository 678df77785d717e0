"""What a server that keeps pages does between the attention of a step and the next step, as cases that can be timed and checked.

Four kinds of case, each one call of an operator:

* ``weights`` -- the attention weight that every cached position received from the call's queries, per key/value head (``esp_paged_key_weights``);
* ``evict``   -- a cache over its budget keeps the positions of the largest accumulated weights and the latest ones (``esp_paged_evict``);
* ``sample``  -- tokens drawn from logits with temperature, top-k, top-p and min-p, from given random numbers (``esp_sample``);
* ``accept``  -- the path of a draft tree whose tokens the model chose, its keys and values moved to their positions (``esp_paged_accept``).

``run`` computes them in elementary torch operations (``own`` false) or through the library (``own`` true).
"""
import math
import random

import numpy as np
import torch

own = False

LLAMA = dict(heads=32, kv_heads=8, head_dim=128)      # head layout of the 8B decoders
TINY = dict(heads=4, kv_heads=2, head_dim=64)         # head layout of the tiny fp32 decoder
VOCAB_LLAMA, VOCAB_QWEN = 128256, 151936


def listed():
    return [
        # one new token of one sequence: the smallest call, latency counts
        dict(name="weights-1-4k", kind="weights", dtype="bf16", page=16, order="head", batch=1, new=1, kv=4096, ragged=False, mask="causal", window=0, last=0, keep=0.0,
             deal=1, **LLAMA),
        # a decode step of 64 sequences of many lengths, added to what the steps before gave
        dict(name="weights-64-ragged", kind="weights", dtype="bf16", page=16, order="head", batch=64, new=1, kv=8192, ragged=True, mask="causal", window=0, last=0, keep=1.0,
             deal=2, **LLAMA),
        # a chunk of a long prompt: what 2048 tokens look at in 8192 positions
        dict(name="weights-chunk-2k", kind="weights", dtype="bf16", page=64, order="head", batch=1, new=2048, kv=8192, ragged=False, mask="causal", window=0, last=0, keep=0.0,
             deal=3, **LLAMA),
        # ragged prompts whose last 32 tokens look back, small heads, pages that end inside every tile
        dict(name="weights-observed", kind="weights", dtype="bf16", page=24, order="token", batch=12, new=500, kv=6001, ragged=True, mask="causal", window=0, last=32, keep=0.5,
             deal=4, heads=16, kv_heads=4, head_dim=64),
        # one position too many in each of 32 sequences: what a decode step at the budget has to do
        dict(name="evict-step-32", kind="evict", dtype="bf16", page=16, order="head", batch=32, kv=2049, budget=2048, recent=256, ragged=False, positions=True, deal=5, **LLAMA),
        # eight long prompts cut to an eighth before their first decode step
        dict(name="evict-8-32k", kind="evict", dtype="bf16", page=64, order="token", batch=8, kv=32768, budget=4096, recent=64, ragged=False, positions=False, deal=6, **LLAMA),
        # sequences of many lengths, some under their budget, full-precision heads of the tiny decoder
        dict(name="evict-fp32-ragged", kind="evict", dtype="fp32", page=24, order="head", batch=13, kv=5001, budget=777, recent=50, ragged=True, positions=True, deal=7, **TINY),
        # one row of logits: the end of a single sequence's step
        dict(name="sample-1", kind="sample", dtype="fp32", rows=1, vocab=VOCAB_LLAMA, mode="all"),
        # the rows of four draft trees, every row's nucleus
        dict(name="sample-trees", kind="sample", dtype="fp32", rows=272, vocab=VOCAB_LLAMA, mode="topp"),
        # a step of many sequences, each with its own settings
        dict(name="sample-256-mixed", kind="sample", dtype="bf16", rows=256, vocab=VOCAB_QWEN, mode="mixed"),
        # one draft tree of 24 rows
        dict(name="accept-1-tree", kind="accept", dtype="fp32", page=16, order="token", batch=1, new=24, kv=1030, ragged=False, deal=8, **TINY),
        # 64 draft trees of up to 64 nodes and 4 probe rows
        dict(name="accept-64-trees", kind="accept", dtype="bf16", page=16, order="head", batch=64, new=68, kv=1100, ragged=True, deal=9, **LLAMA),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng, dtype):
    if dtype == "fp32":
        kv = rng.randint(1, 3)
        return dict(heads=kv * rng.choice([1, 2, 3]), kv_heads=kv, head_dim=rng.choice([32, 64, 128]))
    kv = rng.choice([1, 2, 4, 8])
    return dict(heads=kv * rng.choice([1, 2, 3, 4, 4, 7, 8]), kv_heads=kv, head_dim=rng.choice([64, 128, 128]))


def draw(rng):
    kind = rng.choice(["weights", "weights", "evict", "sample", "sample", "accept"])
    dtype = "bf16" if rng.random() < 0.75 else "fp32"
    if kind == "sample":
        vocab = rng.choice([VOCAB_LLAMA, VOCAB_QWEN, _log(rng, 500, 150000)])
        return dict(kind=kind, dtype=dtype, rows=_log(rng, 1, min(300, 38000000 // vocab)), vocab=vocab,
                    mode=rng.choice(["greedy", "temperature", "topk", "topp", "minp", "all", "mixed", "mixed"]))
    paged = dict(page=rng.choice([16, 16, 32, 64, 128, 24, 8, 17, 200]), order=rng.choice(["head", "token"]), deal=rng.randint(20, 10 ** 6))
    heads = _draw_heads(rng, dtype)
    batch = _log(rng, 1, 32)
    if kind == "accept":
        new = rng.randint(2, 128)
        return dict(kind=kind, dtype=dtype, batch=batch, new=new, kv=new + _log(rng, 1, 1200), ragged=rng.random() < 0.5, **paged, **heads)
    kv = _log(rng, 16, (8192 if dtype == "bf16" else 2048) if batch > 4 else (32768 if dtype == "bf16" else 4096))
    if kind == "evict":
        budget = max(1, min(kv, _log(rng, max(1, kv // 10), kv)) - rng.randint(0, 3))
        return dict(kind=kind, dtype=dtype, batch=batch, kv=kv, budget=budget, recent=rng.choice([0, budget // 16, budget // 4]), ragged=rng.random() < 0.5,
                    positions=rng.random() < 0.6, **paged, **heads)
    mask = rng.choice(["one", "one", "causal", "causal", "tree"])
    new = {"one": 1, "tree": rng.randint(2, 128), "causal": _log(rng, 2, (1200 if dtype == "bf16" else 200) // batch + 2)}[mask]
    kv = max(kv, new)
    window = rng.choice([0, 0, 0, rng.randint(1, kv)]) if mask != "tree" else 0
    last = rng.choice([0, 0, rng.randint(1, 64)])
    return dict(kind=kind, dtype=dtype, batch=batch, new=new, kv=kv, ragged=rng.random() < 0.6, mask="tree" if mask == "tree" else "causal", window=window, last=last,
                keep=rng.choice([0.0, 1.0, 0.9]), **paged, **heads)


# ---------------------------------------------------------------- the batch: lengths and trees follow from the case, the contents from the seed
def _lengths(case):
    """(new tokens, cached positions with them) of every sequence."""
    rng = random.Random(case["deal"])
    n, kv, most = [], [], case.get("new", 1)
    for i in range(case["batch"]):
        ragged = case["ragged"] and i > 0
        n.append(_log(rng, 1, most) if ragged else most)
        kv.append(max(n[-1], _log(rng, max(1, case["kv"] // 8), case["kv"])) if ragged else case["kv"])
    return n, kv


def _budgets(case):
    rng = random.Random(case["deal"] + 2)
    return [max(case["recent"], case["budget"] - rng.randint(0, case["budget"] // 4)) if case["ragged"] and b > 0 else case["budget"] for b in range(case["batch"])]


def _tree(n, rng):
    """Parents (-1: the root) of a random tree of n rows in breadth-first order, depth at most 5, and ancestor-or-self masks."""
    parent, depth, anc = [-1], [0], [1]
    for i in range(1, n):
        p = rng.choice([j for j in range(max(0, i - 24), i) if depth[j] < 5] or [0])
        parent.append(p)
        depth.append(depth[p] + 1)
        anc.append(anc[p] | (1 << i))
    return parent, depth, anc


def _trees(case):
    rng = random.Random(case["deal"] + 1)
    return [_tree(m, rng) for m in _lengths(case)[0]]


def _words(anc):
    signed = lambda w: w - (1 << 64) if w >> 63 else w  # noqa: E731
    return [signed(anc & ((1 << 64) - 1)), signed(anc >> 64)]


def _observed(case):
    """New tokens in front of the observed ones, for every sequence."""
    return [max(0, m - case["last"]) if case["last"] else 0 for m in _lengths(case)[0]]


def _path(parent, depth, rng):
    """Rows of a path from the root that a pass can move again and again: no row goes where another one comes from."""
    for _ in range(40):
        rows, v = [], rng.randrange(len(parent))
        while v > 0:
            rows.append(v)
            v = parent[v]
        rows = rows[::-1]
        if not {i + 1 for i in range(len(rows))} & {r for i, r in enumerate(rows) if r != i + 1}:
            return [0] + rows
    return [0]


# ---------------------------------------------------------------- inputs
def _dt(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _paged(case, g, s):
    """The cache, its page table and the batch's descriptors.  Pages are dealt in a random order, as an allocator hands them out after a while."""
    n, kv = _lengths(case)
    page, heads, d = case["page"], case["kv_heads"], case["head_dim"]
    pages = [-(-t // page) for t in kv]
    total = sum(pages) + 2
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(torch.randint(1 << 30, (1,), generator=g, device="cuda")))).tolist()
    table = torch.full((len(n), max(pages)), -1, dtype=torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = torch.tensor(order[at:at + p], dtype=torch.int32)
        at += p
    shape = (total, heads, page, d) if case["order"] == "head" else (total, page, heads, d)
    for name in ("k", "v"):
        s[name + "_pages"] = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(_dt(case))
    s["slots"] = shape[:3]
    s["table"] = table.cuda()
    s["q_start"] = torch.tensor([0] + n, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32).cuda()
    s["max_new"], s["max_kv"], s["tokens"] = max(n), max(kv), sum(n)
    # where token i of the call stands: its sequence, its place in the block and its position (used by the plain form)
    s["seq"] = torch.tensor([b for b, m in enumerate(n) for _ in range(m)]).cuda()
    s["row"] = torch.tensor([i for m in n for i in range(m)]).cuda()
    s["position"] = torch.tensor([kv[b] - n[b] + i for b, m in enumerate(n) for i in range(m)]).cuda()


def _logits(case, g):
    """Rows as a decoder leaves them: a wide bulk, and a few dozen tokens above it, in some rows so far that they have all of the probability, in some not much more than the bulk."""
    x = 2.0 * torch.randn(case["rows"], case["vocab"], generator=g, device="cuda", dtype=torch.float32)
    few = min(48, case["vocab"] // 8)
    at = torch.randint(0, case["vocab"], (case["rows"], few), generator=g, device="cuda")
    height = 6.0 + 10.0 * torch.rand(case["rows"], 1, generator=g, device="cuda")
    return x.scatter_add_(1, at, 4.0 + height * torch.rand(case["rows"], few, generator=g, device="cuda")).to(_dt(case))


def _settings(case, seed):
    """Temperature, top-k, top-p and min-p of every row; None: the call has no such limit."""
    rng, mode, rows = random.Random(seed), case["mode"], case["rows"]
    want = [rng.choice(["greedy", "temperature", "topk", "topp", "minp", "all"]) if mode == "mixed" else mode for _ in range(rows)]
    t = [0.0 if w == "greedy" else rng.choice([0.6, 0.8, 1.0, 1.2]) for w in want]
    k = [rng.choice([20, 50, 200, 1000]) if w in ("topk", "all") else 0 for w in want]
    p = [rng.choice([0.5, 0.9, 0.95, 0.99]) if w in ("topp", "all") else 1.0 for w in want]
    m = [rng.choice([0.01, 0.05, 0.1]) if w in ("minp", "all") else 0.0 for w in want]
    f = lambda v: torch.tensor(v, dtype=torch.float32).cuda()  # noqa: E731
    return dict(temperature=f(t), top_k=torch.tensor(k, dtype=torch.int32).cuda() if any(k) else None, top_p=f(p) if any(x < 1 for x in p) else None,
                min_p=f(m) if any(m) else None)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "sample":
        s["logits"] = _logits(case, g)
        s["uniform"] = torch.rand(case["rows"], generator=g, device="cuda", dtype=torch.float32)
        s["settings"] = _settings(case, seed)
        s["token"] = torch.empty(case["rows"], dtype=torch.int32, device="cuda")
        s["logprob"] = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
    else:
        _paged(case, g, s)
    if case["kind"] == "weights":
        heads, d = case["heads"], case["head_dim"]
        s["q"] = (2.0 * torch.randn(s["tokens"], heads, d, generator=g, device="cuda", dtype=torch.float32)).to(_dt(case))
        s["before"] = torch.rand(s["slots"], generator=g, device="cuda", dtype=torch.float32)
        s["scores"] = s["before"].clone()
        if case["mask"] == "tree":
            s["anc"] = torch.tensor([_words(a) for _, _, anc in _trees(case) for a in anc], dtype=torch.int64).cuda()
        s["skip"] = torch.tensor(_observed(case)).cuda()
        s["lse"] = _lse(case, s)
    if case["kind"] == "evict":
        # weights as they add up: a few positions have most, some none at all
        x = (2.0 * torch.randn(s["slots"], generator=g, device="cuda", dtype=torch.float32)).exp()
        x = x * (torch.rand(s["slots"], generator=g, device="cuda") > 0.05)
        s["budget"] = torch.tensor(_budgets(case), dtype=torch.int32).cuda()
        if case["positions"]:
            # earlier evictions left `settled` slots with positions of their own, later tokens lie behind them
            kv = _lengths(case)[1]
            settled = torch.tensor([t - 1 - i % max(1, t // 8) if t > 1 else 0 for i, t in enumerate(kv)], dtype=torch.int32).cuda()
            gone = torch.randint(0, 1000, (case["batch"],), generator=g, device="cuda", dtype=torch.int32)
            s["seen"] = s["kv_len"] + gone
            rank = torch.rand(case["batch"], case["kv_heads"], s["max_kv"], generator=g, device="cuda")
            rank = rank.masked_fill(torch.arange(s["max_kv"], device="cuda") >= settled[:, None, None], 2.0).argsort(-1).argsort(-1).int()
            pos = torch.full(s["slots"], -1, dtype=torch.int32, device="cuda")
            _slot_write(case, s, pos, rank, torch.arange(s["max_kv"], device="cuda") < settled[:, None])
            s["start"] = torch.cat([x.view(torch.int32).flatten(), pos.flatten(), settled])
        else:
            s["start"] = x.view(torch.int32).flatten()
        # what a call changes beside the pages, in one buffer, so that a pass can begin where the first one began
        s["now"] = s["start"].clone()
        n = x.numel()
        s["scores"] = s["now"][:n].view(torch.float32).view(s["slots"])
        s["positions"] = s["now"][n:2 * n].view(s["slots"]) if case["positions"] else None
        s["settled"] = s["now"][2 * n:] if case["positions"] else None
        s["kv_out"] = torch.empty_like(s["kv_len"])
    if case["kind"] == "accept":
        rng = random.Random(seed)
        parents, drafted, chosen = [], [], []
        for parent, depth, _ in _trees(case):
            probes = 4 if len(parent) > 8 else 0                      # the last rows are probes, no drafts: they hang on nothing
            parent, depth = parent[:len(parent) - probes], depth[:len(parent) - probes]
            token = [rng.randrange(VOCAB_LLAMA) for _ in parent]
            choice = [rng.randrange(VOCAB_LLAMA) for _ in parent]
            path = _path(parent, depth, rng)
            for a, b in zip(path, path[1:]):
                choice[a] = token[b]
            parents += parent + [-1] * probes
            drafted += token + [-1] * probes
            chosen += choice + [0] * probes
        s["parents"], s["drafted"], s["chosen"] = (torch.tensor(x, dtype=torch.int32).cuda() for x in (parents, drafted, chosen))
        s["out_tokens"], s["out_rows"] = (torch.empty(case["batch"], s["max_new"], dtype=torch.int32, device="cuda") for _ in range(2))
        s["n_out"], s["kv_out"] = torch.empty_like(s["kv_len"]), torch.empty_like(s["kv_len"])
    if own:
        import paper_2603_17942_b200 as P
        s["P"] = P
        if case["kind"] == "sample":
            nb = P.esp_sample_scratch_bytes(case["rows"], case["vocab"])
        else:
            s["cache"] = P.PagedCache(s["k_pages"], s["v_pages"], order=case["order"])
            s["batch"] = P.PagedBatch(s["q_start"], s["kv_len"], s["table"], s["max_new"])
            nb = 0
        if case["kind"] == "weights":
            nb = P.esp_paged_key_weights_scratch_bytes(s["tokens"], case["heads"], case["head_dim"])
        if case["kind"] == "evict":
            nb = P.esp_paged_evict_scratch_bytes(case["batch"], case["kv_heads"], s["max_kv"])
        if case["kind"] in ("weights", "evict"):
            s["slot_scores"] = P.PagedSlots(s["scores"], order=case["order"])
            s["slot_positions"] = P.PagedSlots(s["positions"], order=case["order"]) if s.get("positions") is not None else None
        s["scratch"], s["scratch_bytes"] = torch.empty(max(nb, 1), dtype=torch.uint8, device="cuda"), nb
    return s


# ---------------------------------------------------------------- the operators
def run(s):
    case = s["case"]
    if own:
        P, stream = s["P"], torch.cuda.current_stream().cuda_stream
        if case["kind"] == "weights":
            if case["keep"]:
                s["scores"].copy_(s["before"])
            P.esp_paged_key_weights(s["cache"], s["batch"], s["q"], s["lse"], s["slot_scores"], s["scratch"], s["scratch_bytes"], anc=s.get("anc"), window=case["window"],
                                    last=case["last"], keep=case["keep"], stream=stream)
            return s["scores"]
        if case["kind"] == "evict":
            s["now"].copy_(s["start"])
            P.esp_paged_evict(s["cache"], s["batch"], s["slot_scores"], s["budget"], s["kv_out"], s["scratch"], s["scratch_bytes"], recent=case["recent"],
                              positions=s["slot_positions"], settled=s["settled"], seen=s.get("seen"), stream=stream)
            return (s["kv_out"], s["k_pages"], s["v_pages"], s["scores"]) + ((s["positions"], s["settled"]) if case["positions"] else ())
        if case["kind"] == "sample":
            P.esp_sample(s["logits"], s["uniform"], s["token"], s["scratch"], s["scratch_bytes"], logprob=s["logprob"], stream=stream, **s["settings"])
            return s["token"], s["logprob"]
        P.esp_paged_accept(s["cache"], s["batch"], s["parents"], s["drafted"], s["chosen"], s["out_tokens"], s["n_out"], s["kv_out"], rows=s["out_rows"], stream=stream)
        return s["n_out"], s["kv_out"], s["out_tokens"], s["out_rows"], s["k_pages"], s["v_pages"]
    if case["kind"] == "weights":
        s["scores"].copy_(s["before"])
        return _weights(case, s)
    if case["kind"] == "evict":
        s["now"].copy_(s["start"])
        return _evict(case, s)
    if case["kind"] == "sample":
        return _sample(s["logits"], s["uniform"], **s["settings"])
    return _accept(case, s)


def _slot_read(case, s, x):
    """[pages ...] -> [batch, kv_heads, positions] (or [..., head_dim]) of every sequence, padded to the longest."""
    y = x[s["table"].long().clamp(min=0)]
    y = y.transpose(2, 3) if case["order"] == "head" else y
    return y.reshape(len(y), -1, *y.shape[3:])[:, :s["max_kv"]].transpose(1, 2)


def _slot_write(case, s, x, y, where):
    """y [batch, kv_heads, positions] into the pages at the positions that `where` [batch, positions] marks."""
    b, p = where.nonzero(as_tuple=True)
    page, slot = s["table"][b, p // case["page"]].long(), p % case["page"]
    if case["order"] == "head":
        x[page, :, slot] = y[b, :, p]
    else:
        x[page, slot] = y[b, :, p]


def _scores(case, s):
    """Scaled products of every query with its sequence's keys and what the masks leave: [batch, kv_heads, group, new, positions], and which of them count."""
    b, n, t = case["batch"], s["max_new"], s["max_kv"]
    hk, g, d = case["kv_heads"], case["heads"] // case["kv_heads"], case["head_dim"]
    key = torch.arange(t, device="cuda")
    k = _slot_read(case, s, s["k_pages"]).float()
    q = torch.zeros(b, n, hk, g, d, device="cuda")
    q[s["seq"], s["row"]] = s["q"].float().reshape(-1, hk, g, d)
    x = (q.permute(0, 2, 3, 1, 4).reshape(b, hk, g * n, d) @ k.transpose(2, 3)).view(b, hk, g, n, t) / math.sqrt(d)
    at = torch.full((b, n), -1, device="cuda")
    at[s["seq"], s["row"]] = s["position"]
    first = (s["kv_len"] - s["q_start"].diff())[:, None, None]       # position of each sequence's first new token
    if case["mask"] == "tree":
        anc = torch.zeros(b, n, 2, dtype=torch.int64, device="cuda")
        anc[s["seq"], s["row"]] = s["anc"]
        place = (key - first).clamp(0, 127)
        bit = torch.where(place < 64, anc[..., 0:1] >> (place % 64), anc[..., 1:2] >> (place % 64)) & 1
        seen = (key < first) | ((bit == 1) & (key < s["kv_len"][:, None, None]))
    else:
        seen = key <= at[..., None]
    if case["window"]:
        seen = seen & (key > at[..., None] - case["window"])
    return x, (seen & (at >= 0)[..., None])[:, None, None]


def _lse(case, s):
    x, seen = _scores(case, s)
    return torch.where(seen, x, -math.inf).logsumexp(-1).permute(0, 3, 1, 2)[s["seq"], s["row"]].reshape(-1, case["heads"]).contiguous()


def _weights(case, s):
    b, n, t = case["batch"], s["max_new"], s["max_kv"]
    hk, g = case["kv_heads"], case["heads"] // case["kv_heads"]
    x, seen = _scores(case, s)
    lse = torch.zeros(b, n, hk, g, device="cuda")
    lse[s["seq"], s["row"]] = s["lse"].view(-1, hk, g)
    seen = seen & (torch.arange(n, device="cuda") >= s["skip"][:, None])[:, None, None, :, None]
    w = torch.where(seen, (x - lse.permute(0, 2, 3, 1)[..., None]).exp(), 0.0).sum((2, 3))
    key = torch.arange(t, device="cuda")
    if case["keep"]:                                                  # the new tokens' own slots begin at zero
        old = key < (s["kv_len"] - s["q_start"].diff())[:, None]
        w = w + torch.where(old[:, None], case["keep"] * _slot_read(case, s, s["scores"]), 0.0)
    _slot_write(case, s, s["scores"], w, key < s["kv_len"][:, None])
    return s["scores"]


def _evict(case, s):
    key, kv = torch.arange(s["max_kv"], device="cuda"), s["kv_len"][:, None, None]
    x = _slot_read(case, s, s["scores"])
    seen = s["seen"][:, None, None] if case["positions"] else kv
    pos = (seen - kv + key).expand(x.shape)
    if case["positions"]:
        pos = torch.where(key < s["settled"][:, None, None], _slot_read(case, s, s["positions"]), pos)
    full = (kv > s["budget"][:, None, None])
    x = torch.where(pos >= seen - case["recent"], math.inf, torch.where(x.isnan(), -math.inf, x))
    order = torch.where(key < kv, x, -math.inf).sort(dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, key.expand(x.shape))
    budget = s["budget"][:, None, None]
    kept = rank < budget
    source, hole = full & kept & (key >= budget), full & ~kept & (key < budget)
    if case["positions"]:
        _slot_write(case, s, s["positions"], pos.int(), (full & (key < budget))[:, 0])
    b, h, i = source.nonzero(as_tuple=True)
    _, _, j = hole.nonzero(as_tuple=True)
    place = lambda p: (s["table"][b, p // case["page"]].long(), h, p % case["page"]) if case["order"] == "head" else \
        (s["table"][b, p // case["page"]].long(), p % case["page"], h)  # noqa: E731
    s["k_pages"][place(j)] = s["k_pages"][place(i)]
    s["v_pages"][place(j)] = s["v_pages"][place(i)]
    s["scores"][place(j)] = s["scores"][place(i)]
    kv_out = torch.minimum(s["kv_len"], s["budget"])
    if not case["positions"]:
        return kv_out, s["k_pages"], s["v_pages"], s["scores"]
    s["positions"][place(j)] = pos[b, h, i].int()
    s["settled"].copy_(torch.where(full[:, 0, 0], s["budget"], s["settled"]))
    return kv_out, s["k_pages"], s["v_pages"], s["scores"], s["positions"], s["settled"]


def _sample(logits, uniform, temperature, top_k, top_p, min_p):
    rows, vocab = logits.shape
    x, index = logits.double().sort(dim=-1, descending=True, stable=True)
    t = temperature.double()[:, None]
    w = ((x - x[:, :1]) / torch.where(t > 0, t, 1.0)).exp()
    rank = torch.arange(vocab, device="cuda")
    kept = (rank == 0) | (t > 0)
    if top_k is not None:
        kept = kept & ((top_k[:, None] <= 0) | (rank < top_k[:, None]))
    if top_p is not None:
        y = torch.where(kept, w, 0.0)
        before = y.cumsum(-1) - y
        kept = kept & ((top_p[:, None] >= 1) | (before < top_p.double()[:, None] * y.sum(-1, keepdim=True)))
    if min_p is not None:
        kept = kept & (w >= min_p.double()[:, None])
    w = torch.zeros_like(w).scatter_(-1, index, torch.where(kept, w, 0.0))
    upto = w.cumsum(-1)
    token = (upto > uniform.double()[:, None] * upto[:, -1:]).int().argmax(-1)
    return token.int(), (w.gather(-1, token[:, None])[:, 0] / upto[:, -1]).log().float()


def _accept(case, s):
    """Depth by depth: every sequence's next row is the first child of its row that carries the token chosen there."""
    b, n, top = case["batch"], s["max_new"], 5
    pad = lambda x, none: torch.full((b, n), none, device="cuda").index_put_((s["seq"], s["row"]), x.long())  # noqa: E731
    parents, drafted, chosen = pad(s["parents"], -2), pad(s["drafted"], -1), pad(s["chosen"], -1)
    at = torch.zeros(b, 1, dtype=torch.long, device="cuda")
    tokens, rows, alive = [], [], torch.ones(b, 1, dtype=torch.bool, device="cuda")
    for _ in range(min(n, top + 1)):
        want = chosen.gather(1, at)
        tokens.append(torch.where(alive, want, -1))
        rows.append(torch.where(alive, at, -1))
        fits = (parents == at) & (drafted == want)
        alive = alive & fits.any(1, keepdim=True)
        at = torch.where(alive, fits.int().argmax(1, keepdim=True), at)
    fill = lambda x: torch.cat(x + [torch.full((b, n - len(x)), -1, device="cuda")], 1).int()  # noqa: E731
    tokens, rows = fill(tokens), fill(rows)
    count = (rows >= 0).sum(1).int()
    first = s["kv_len"] - s["q_start"].diff()
    i, j = ((rows > 0) & (rows != torch.arange(n, device="cuda"))).nonzero(as_tuple=True)
    source, target = first[i] + rows[i, j], first[i] + j
    place = lambda p: (s["table"][i, p // case["page"]].long(), p % case["page"])  # noqa: E731
    for x in (s["k_pages"], s["v_pages"]):
        x = x.transpose(1, 2) if case["order"] == "head" else x
        x[place(target)] = x[place(source)]
    return count, first + count, tokens, rows, s["k_pages"], s["v_pages"]


# ---------------------------------------------------------------- what an operator cannot do without, and its results in 64 bits
def work(case):
    if case["kind"] == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * (4 if case["dtype"] == "fp32" else 2) + 12), "flops": 2 * case["rows"] * case["vocab"]}
    size, d, hk = 4 if case["dtype"] == "fp32" else 2, case["head_dim"], case["kv_heads"]
    n, kv = _lengths(case)
    if case["kind"] == "weights":
        pairs = keys = 0
        trees = _trees(case) if case["mask"] == "tree" else None
        for b, (m, t, skip) in enumerate(zip(n, kv, _observed(case))):
            if trees:
                pairs += (m - skip) * (t - m) + sum(bin(a).count("1") for a in trees[b][2][skip:])
                keys += t
            else:
                w = case["window"] or t
                pairs += sum(min(w, t - m + i + 1) for i in range(skip, m))
                keys += min(t, w + m - skip - 1)
        tokens = sum(n) - sum(_observed(case))
        return {"bytes": keys * hk * d * size + tokens * case["heads"] * (d * size + 4) + sum(kv) * hk * (8 if case["keep"] else 4),
                "flops": 2 * d * case["heads"] * pairs}
    if case["kind"] == "evict":
        bytes_ = 0
        for t, most in zip(kv, _budgets(case)):
            if t > most:
                moved = (t - most) * min(1.0, most / t)                # slots behind the budget that are kept, as often as any other
                bytes_ += hk * (t * (8 if case["positions"] else 4) + moved * (4 * d * size + 8))
        return {"bytes": bytes_ + 12 * case["batch"], "flops": hk * sum(kv)}
    return {"bytes": sum(n) * 12 + case["batch"] * (8 * case["new"] + 16 + 2 * 4 * hk * d * size), "flops": sum(n)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(case, s)
    n, kv = _lengths(case)
    table = s["table"].cpu()
    d, hk, order = case["head_dim"], case["kv_heads"], case["order"]
    group = case["heads"] // hk

    def slots(b, p):
        p = torch.as_tensor(p)
        return table[b][torch.div(p, case["page"], rounding_mode="floor")].long().cuda(), (p % case["page"]).cuda()

    if case["kind"] == "weights":
        out, at = s["before"].double(), 0
        trees = _trees(case) if case["mask"] == "tree" else None
        for b, (m, t, skip) in enumerate(zip(n, kv, _observed(case))):
            page, slot = slots(b, torch.arange(t))
            i, j = torch.arange(t - m + skip, t, device="cuda")[:, None], torch.arange(t, device="cuda")[None]
            hidden = j > i
            if case["window"]:
                hidden = hidden | (i - j >= case["window"])
            if trees:
                rows = torch.tensor([[bool((a >> c) & 1) for c in range(m)] for a in trees[b][2][skip:]], device="cuda").view(m - skip, m)
                hidden = torch.cat([torch.zeros(m - skip, t - m, dtype=torch.bool, device="cuda"), ~rows], 1)
            for h in range(hk):
                k = (s["k_pages"][page, h, slot] if order == "head" else s["k_pages"][page, slot, h]).double()
                total = torch.zeros(t, dtype=torch.float64, device="cuda")
                for e in range(h * group, (h + 1) * group):
                    logits = torch.einsum("id,jd->ij", s["q"][at + skip:at + m, e].double(), k).mul_(d ** -0.5)
                    total += logits.sub_(s["lse"][at + skip:at + m, e].double()[:, None]).masked_fill_(hidden, -math.inf).exp().sum(0)
                view = out[:, h] if order == "head" else out[:, :, h]
                if case["keep"]:
                    total[:t - m] += case["keep"] * view[page, slot][:t - m]
                view[page, slot] = total
            at += m
        return out
    if case["kind"] == "evict":
        scores, budgets = s["scores"].cpu().numpy(), _budgets(case)
        where = s["positions"].cpu().numpy() if case["positions"] else None
        settled = s["settled"].tolist() if case["positions"] else [0] * len(kv)
        seen = s["seen"].tolist() if case["positions"] else kv
        ends = list(settled)
        for b, t in enumerate(kv):
            keep = budgets[b]
            if t <= keep:
                continue
            ends[b] = keep
            p = np.arange(t)
            page, slot = table[b].numpy()[p // case["page"]], p % case["page"]
            for h in range(hk):
                at = (page, h, slot) if order == "head" else (page, slot, h)
                x, pos = scores[at], seen[b] - t + p
                if where is not None:
                    pos = np.where(p < settled[b], where[at], pos)
                rank = np.lexsort((p, -np.where(pos >= seen[b] - case["recent"], np.inf, x)))
                best = set(rank[:keep].tolist())
                source = np.array([i for i in range(keep, t) if i in best], dtype=np.int64)
                target = np.array([i for i in range(keep) if i not in best], dtype=np.int64)
                new, newpos = x[:keep].copy(), pos[:keep].copy()
                new[target], newpos[target] = x[source], pos[source]
                front = tuple(a[:keep] if isinstance(a, np.ndarray) else a for a in at)
                scores[front] = new
                if where is not None:
                    where[front] = newpos
                (fp, fs), (tp, ts) = slots(b, source), slots(b, target)
                for pages in (s["k_pages"], s["v_pages"]):
                    view = pages[:, h] if order == "head" else pages[:, :, h]
                    view[tp, ts] = view[fp, fs]
        out = (torch.tensor([min(t, m) for t, m in zip(kv, budgets)], dtype=torch.int32), s["k_pages"], s["v_pages"], torch.from_numpy(scores))
        return out + ((torch.from_numpy(where), torch.tensor(ends, dtype=torch.int32)) if case["positions"] else ())
    parents, drafted, chosen = (s[x].tolist() for x in ("parents", "drafted", "chosen"))
    tokens, rows = (torch.full((len(n), max(n)), -1, dtype=torch.int32) for _ in range(2))
    count, at = [], 0
    for b, (m, t) in enumerate(zip(n, kv)):
        path, row = [], 0
        while row is not None:
            path.append(row)
            want = chosen[at + row]
            row = next((i for i in range(m) if parents[at + i] == row and drafted[at + i] == want), None)
        tokens[b, :len(path)] = torch.tensor([chosen[at + r] for r in path])
        rows[b, :len(path)] = torch.tensor(path)
        count.append(len(path))
        (fp, fs), (tp, ts) = slots(b, [t - m + r for r in path]), slots(b, [t - m + i for i in range(len(path))])
        for pages in (s["k_pages"], s["v_pages"]):
            view = pages.transpose(1, 2) if order == "head" else pages
            view[tp, ts] = view[fp, fs]
        at += m
    return (torch.tensor(count, dtype=torch.int32), torch.tensor([t - m + c for t, m, c in zip(kv, n, count)], dtype=torch.int32), tokens, rows, s["k_pages"], s["v_pages"])


def _exact_sample(case, s):
    token, logprob = [], []
    host = lambda name, none: s["settings"][name].cpu().numpy() if s["settings"][name] is not None else [none] * case["rows"]  # noqa: E731
    t, k, p, m, u = host("temperature", 1.0), host("top_k", 0), host("top_p", 1.0), host("min_p", 0.0), s["uniform"].cpu().numpy()
    for r in range(case["rows"]):
        x = s["logits"][r].double().cpu().numpy()
        if t[r] == 0:
            token.append(int(x.argmax()))
            logprob.append(0.0)
            continue
        w = np.exp((x - x.max()) / np.float64(t[r]))
        order = np.argsort(-x, kind="stable")[:k[r] if k[r] > 0 else len(x)]
        if p[r] < 1:
            mass = np.concatenate([[0.0], np.cumsum(w[order])])
            order = order[:np.searchsorted(mass[:-1], np.float64(p[r]) * mass[-1], side="left")]
        order = np.sort(order[w[order] >= np.float64(m[r])])
        upto = np.cumsum(w[order])
        i = int(np.searchsorted(upto, np.float64(u[r]) * upto[-1], side="right"))
        token.append(int(order[i]))
        logprob.append(math.log(w[order[i]] / upto[-1]))
    return torch.tensor(token, dtype=torch.int32), torch.tensor(logprob, dtype=torch.float64)
