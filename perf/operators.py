"""The paged-cache operators as cases that can be timed and checked: what a serving loop does around the decode-and-verify block
when keys and values live in pages.

Three kinds of case, each one call of an operator:

* ``norm_rope`` -- per-head RMSNorm of queries and keys with the position rotation (``esp_qk_norm_rope``);
* ``append``    -- the same on the way into the pages of a cache, values along with it (``esp_paged_append``);
* ``attention`` -- new tokens of a ragged batch over the pages (``esp_paged_attention``): causal, with a sliding window, or with the
                   ancestor masks of a draft tree.

``run`` computes them in elementary torch operations (``own`` false) or through the library (``own`` true).
"""
import math
import random

import torch

own = False

LLAMA = dict(heads=32, kv_heads=8, head_dim=128)      # head layout of the 8B decoders
TINY = dict(heads=4, kv_heads=2, head_dim=64)         # head layout of the tiny fp32 decoder
ROPE_LLAMA = dict(base=500000.0, rotary=128, interleaved=False, scaling="none", factor=1.0, norm=False)
ROPE_QWEN = dict(base=1000000.0, rotary=128, interleaved=False, scaling="none", factor=1.0, norm=True)
ORIGINAL = 8192        # positions the scaled frequencies were made for
EPS = 1e-6


def listed():
    return [
        # one new token of one sequence: the smallest call, latency counts
        dict(name="norm-rope-1", kind="norm_rope", dtype="bf16", tokens=1, far=4096, **LLAMA, **ROPE_QWEN),
        # a long prompt's queries and keys, as views into one projection output
        dict(name="norm-rope-8192", kind="norm_rope", dtype="bf16", tokens=8192, far=32768, **LLAMA, **ROPE_QWEN),
        # full-precision heads, neighbours as pairs, half of the head rotated, positions far beyond the original range
        dict(name="rope-fp32-partial", kind="norm_rope", dtype="fp32", tokens=1777, far=1000000, **TINY, base=10000.0, rotary=32, interleaved=True,
             scaling="linear", factor=8.0, norm=False),
        # a decode step of 64 sequences: one token of each goes into its page
        dict(name="append-decode-64", kind="append", dtype="bf16", page=16, order="head", batch=64, new=1, kv=512, deal=1, **LLAMA, **ROPE_QWEN),
        # chunks of four prompts in one call, scaled frequencies, pages of 64 tokens
        dict(name="append-chunks", kind="append", dtype="bf16", page=64, order="token", batch=4, new=2048, kv=4000, deal=2, **LLAMA,
             **{**ROPE_LLAMA, "scaling": "rotations", "factor": 8.0}),
        # one sequence, one token: the smallest attention call
        dict(name="attend-1-4k", kind="attention", dtype="bf16", page=16, order="head", batch=1, new=1, kv=4096, ragged=False, mask="causal", window=0, deal=3, **LLAMA),
        # a decode step of 64 sequences of many lengths
        dict(name="attend-64-ragged", kind="attention", dtype="bf16", page=16, order="head", batch=64, new=1, kv=8192, ragged=True, mask="causal", window=0, deal=4, **LLAMA),
        # the longest contexts: eight sequences of 32k
        dict(name="attend-8-32k", kind="attention", dtype="bf16", page=64, order="token", batch=8, new=1, kv=32768, ragged=False, mask="causal", window=0, deal=5, **LLAMA),
        # draft trees of 64 nodes and 4 probe rows over 4k positions each
        dict(name="attend-trees", kind="attention", dtype="bf16", page=16, order="head", batch=4, new=68, kv=4164, ragged=False, mask="tree", window=0, deal=6, **LLAMA),
        # a chunk of a long prompt: 2048 tokens behind 6144 cached ones
        dict(name="attend-chunk-2k", kind="attention", dtype="bf16", page=64, order="head", batch=1, new=2048, kv=8192, ragged=False, mask="causal", window=0, deal=7, **LLAMA),
        # prompts' chunks and single tokens in one call, small heads, a sliding window, pages that end inside every tile
        dict(name="attend-mixed-window", kind="attention", dtype="bf16", page=24, order="token", batch=12, new=500, kv=3001, ragged=True, mask="causal", window=1000, deal=8,
             heads=16, kv_heads=4, head_dim=64),
        # full-precision heads of the tiny decoder, chunks of several lengths
        dict(name="attend-fp32", kind="attention", dtype="fp32", page=16, order="head", batch=5, new=100, kv=777, ragged=True, mask="causal", window=0, deal=9, **TINY),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng, dtype):
    if dtype == "fp32":
        kv = rng.randint(1, 3)
        return dict(heads=kv * rng.choice([1, 2, 3]), kv_heads=kv, head_dim=rng.choice([32, 64, 128]))
    kv = rng.choice([1, 2, 4, 8])
    return dict(heads=kv * rng.choice([1, 2, 3, 4, 4, 7, 8]), kv_heads=kv, head_dim=rng.choice([64, 128, 128]))


def _draw_rope(rng, head_dim):
    scaling = rng.choice(["none", "none", "linear", "base", "rotations", "index"])
    return dict(base=rng.choice([10000.0, 500000.0, 1000000.0]), rotary=rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4 + 4]),
                interleaved=rng.random() < 0.4, scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]), norm=rng.random() < 0.5)


def draw(rng):
    kind = rng.choice(["norm_rope", "append", "attention", "attention", "attention"])
    dtype = "bf16" if rng.random() < 0.8 else "fp32"
    heads = _draw_heads(rng, dtype)
    if kind == "norm_rope":
        return dict(kind=kind, dtype=dtype, tokens=_log(rng, 1, 4096), far=_log(rng, 64, 1 << 20), **heads, **_draw_rope(rng, heads["head_dim"]))
    paged = dict(page=rng.choice([16, 16, 32, 64, 128, 24, 8, 17, 200]), order=rng.choice(["head", "token"]), deal=rng.randint(10, 10 ** 6))
    if kind == "append":
        batch = _log(rng, 1, 64)
        new = rng.choice([1, _log(rng, 1, 2048 // batch + 1)])
        return dict(kind=kind, dtype=dtype, batch=batch, new=new, kv=max(new, _log(rng, 16, 600)), **paged, **heads, **_draw_rope(rng, heads["head_dim"]))
    mask = rng.choice(["one", "one", "causal", "causal", "tree"])
    batch = _log(rng, 1, 32)
    kv = _log(rng, 16, (8192 if dtype == "bf16" else 2048) if batch > 4 else (32768 if dtype == "bf16" else 4096))
    new = {"one": 1, "tree": rng.randint(2, 128), "causal": _log(rng, 2, (1200 if dtype == "bf16" else 200) // batch + 2)}[mask]
    kv = max(kv, new)
    window = rng.choice([0, 0, 0, rng.randint(1, kv)]) if mask != "tree" else 0
    return dict(kind=kind, dtype=dtype, batch=batch, new=new, kv=kv, ragged=rng.random() < 0.6, mask="tree" if mask == "tree" else "causal", window=window, **paged, **heads)


# ---------------------------------------------------------------- the batch: lengths follow from the case, the contents from the seed
def _lengths(case):
    """(new tokens, cached positions with them) of every sequence."""
    rng = random.Random(case["deal"])
    n, kv = [], []
    for i in range(case["batch"]):
        ragged = case.get("ragged", case["new"] > 1) and i > 0
        n.append(_log(rng, 1, case["new"]) if ragged else case["new"])
        kv.append(max(n[-1], _log(rng, max(1, case["kv"] // 8), case["kv"])) if ragged else case["kv"])
    return n, kv


def _tree_anc(n, rng):
    """Ancestor-or-self masks of a random tree of n rows in breadth-first order, depth at most 5, as [n][2] words of 64 bits."""
    depth, anc = [0], [1]
    for i in range(1, n):
        p = rng.choice([j for j in range(max(0, i - 24), i) if depth[j] < 5] or [0])
        depth.append(depth[p] + 1)
        anc.append(anc[p] | (1 << i))
    signed = lambda w: w - (1 << 64) if w >> 63 else w  # noqa: E731
    return [[signed(a & ((1 << 64) - 1)), signed(a >> 64)] for a in anc], [bin(a).count("1") for a in anc]


def _anc_of(case, n):
    rng = random.Random(case["deal"] + 1)
    return [_tree_anc(m, rng) for m in n]


def _visible(case):
    """(query-key pairs, distinct keys) that the masks leave, summed over the sequences."""
    n, kv = _lengths(case)
    pairs = keys = 0
    anc = _anc_of(case, n) if case["mask"] == "tree" else None
    for b, (m, t) in enumerate(zip(n, kv)):
        w = case["window"] or t
        if anc:
            pairs += m * (t - m) + sum(anc[b][1])
        else:
            pairs += sum(min(w, t - m + i + 1) for i in range(m))
        keys += min(t, w + m - 1)
    return pairs, keys


# ---------------------------------------------------------------- inputs
def _dt(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _paged(case, g, s):
    """The cache, its page table and the batch's descriptors.  Pages are dealt in a random order, as an allocator hands them out after a while."""
    n, kv = _lengths(case)
    page, heads, d = case["page"], case["kv_heads"], case["head_dim"]
    pages = [-(-t // page) for t in kv]
    spare = 2
    total = sum(pages) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(torch.randint(1 << 30, (1,), generator=g, device="cuda")))).tolist()
    table = torch.full((len(n), max(pages)), -1, dtype=torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = torch.tensor(order[at:at + p], dtype=torch.int32)
        at += p
    shape = (total, heads, page, d) if case["order"] == "head" else (total, page, heads, d)
    for name in ("k", "v"):
        s[name + "_pages"] = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(_dt(case))
    s["table"] = table.cuda()
    s["q_start"] = torch.tensor([0] + n, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32).cuda()
    s["max_new"], s["max_kv"], s["tokens"] = max(n), max(kv), sum(n)
    # where token i of the call stands: its sequence, its place in the block and its position (used by the plain form)
    seq = torch.tensor([b for b, m in enumerate(n) for _ in range(m)])
    row = torch.tensor([i for m in n for i in range(m)])
    s["seq"], s["row"] = seq.cuda(), row.cuda()
    s["position"] = torch.tensor([kv[b] - n[b] + i for b, m in enumerate(n) for i in range(m)]).cuda()
    if case.get("mask") == "tree":
        s["anc"] = torch.tensor([w for words, _ in _anc_of(case, n) for w in words], dtype=torch.int64).cuda()


def _rope_cfg(P, case):
    return P.rope_cfg(case["rotary"], base=case["base"], interleaved=case["interleaved"], scaling=case["scaling"], factor=case["factor"],
                      original_len=ORIGINAL, amplitude=_amplitude(case))


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "index" else 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    heads, kvh, d = case["heads"], case["kv_heads"], case["head_dim"]
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    if case["kind"] != "norm_rope":
        _paged(case, g, s)
    else:
        s["tokens"] = case["tokens"]
        s["positions"] = torch.randint(0, case["far"], (case["tokens"],), generator=g, device="cuda", dtype=torch.int32)
    tokens = s["tokens"]
    # queries, keys and values are views into one projection output, as a fused projection leaves them
    qkv = randn(tokens, heads + 2 * kvh, d).to(_dt(case))
    s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kvh], qkv[:, heads + kvh:]
    if case["kind"] == "attention":
        s["q"] = (2.0 * randn(tokens, heads, d)).to(_dt(case))
        s["out"] = torch.empty_like(s["q"])
    else:
        s["q_gain"], s["k_gain"] = ((1.0 + 0.1 * randn(d)).to(_dt(case)) if case["norm"] else None for _ in range(2))
        s["q_out"] = torch.empty(tokens, heads, d, dtype=_dt(case), device="cuda")
        s["k_out"] = torch.empty(tokens, kvh, d, dtype=_dt(case), device="cuda")
    if own:
        import paper_2603_17942_b200 as P
        s["P"] = P
        if case["kind"] != "norm_rope":
            s["cache"] = P.PagedCache(s["k_pages"], s["v_pages"], order=case["order"])
            s["batch"] = P.PagedBatch(s["q_start"], s["kv_len"], s["table"], s["max_new"])
        if case["kind"] == "attention":
            nb = P.esp_paged_attention_scratch_bytes(heads, d)
            s["scratch"], s["scratch_bytes"] = torch.empty(nb, dtype=torch.uint8, device="cuda"), nb
        else:
            s["rope"] = _rope_cfg(P, case)
            s["rope_table"] = torch.empty(P.esp_rope_table_bytes(s["rope"]), dtype=torch.uint8, device="cuda")
            P.esp_rope_table(s["rope"], s["rope_table"])
    return s


# ---------------------------------------------------------------- the operators
def run(s):
    case = s["case"]
    if own:
        P, stream = s["P"], torch.cuda.current_stream().cuda_stream
        if case["kind"] == "norm_rope":
            P.esp_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["rope"], s["rope_table"], s["positions"], q_gain=s["q_gain"], k_gain=s["k_gain"],
                               eps=EPS, stream=stream)
            return s["q_out"], s["k_out"]
        if case["kind"] == "append":
            P.esp_paged_append(s["cache"], s["batch"], s["k"], s["v"], s["rope"], s["rope_table"], k_gain=s["k_gain"], q=s["q"], q_out=s["q_out"],
                               q_gain=s["q_gain"], eps=EPS, stream=stream)
            return s["q_out"], s["k_pages"], s["v_pages"]
        P.esp_paged_attention(s["cache"], s["batch"], s["q"], s["out"], s["scratch"], s["scratch_bytes"], anc=s.get("anc"), window=case["window"], stream=stream)
        return s["out"]
    if case["kind"] == "norm_rope":
        return _norm_rope(case, s["q"], s["positions"], s["q_gain"]), _norm_rope(case, s["k"], s["positions"], s["k_gain"])
    if case["kind"] == "append":
        page = s["table"][s["seq"], s["position"] // case["page"]].long()
        slot = s["position"] % case["page"]
        k, v = s["k_pages"].clone(), s["v_pages"].clone()
        new = _norm_rope(case, s["k"], s["position"], s["k_gain"])
        if case["order"] == "head":
            k[page, :, slot], v[page, :, slot] = new, s["v"]
        else:
            k[page, slot], v[page, slot] = new, s["v"]
        return _norm_rope(case, s["q"], s["position"], s["q_gain"]), k, v
    return _attention(case, s)


def _frequencies(case):
    """Radians per position of the rotated pairs, in 64 bits: the geometric series, changed for long contexts."""
    r, base, factor = case["rotary"], case["base"], case["factor"]
    i = torch.arange(r // 2, device="cuda", dtype=torch.float64)
    if case["scaling"] == "base":                       # the base grown so that the slowest pair turns `factor` times slower
        base = base * factor ** (r / (r - 2))
    f = base ** (-2.0 * i / r)
    if case["scaling"] == "linear":                     # every pair slower
        return f / factor
    if case["scaling"] == "rotations":                  # pairs that turn less than once in the original length slower, more than 4 times kept, linear between
        keep = ((ORIGINAL * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep
    if case["scaling"] == "index":                      # linear in the pair's index between those that turn 32 times and once
        at = lambda turns: r * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep
    return f


def _norm_rope(case, x, positions, gain):
    y = x.float()
    if gain is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * gain.float()
    angle = positions.double()[:, None, None] * _frequencies(case)
    c, s = (angle.cos() * _amplitude(case)).float(), (angle.sin() * _amplitude(case)).float()
    r = case["rotary"]
    out = y.clone()
    if case["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        out[..., 0:r:2], out[..., 1:r:2] = a * c - b * s, b * c + a * s
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        out[..., :r // 2], out[..., r // 2:r] = a * c - b * s, b * c + a * s
    return out.to(x.dtype)


def _attention(case, s):
    """Every sequence padded to the longest: gather the pages, scores, mask, softmax, values."""
    b, n, t = case["batch"], s["max_new"], s["max_kv"]
    hk, g, d = case["kv_heads"], case["heads"] // case["kv_heads"], case["head_dim"]
    pages = s["table"].long().clamp(min=0)
    gather = lambda x: (x[pages].transpose(2, 3) if case["order"] == "head" else x[pages]).reshape(b, -1, hk, d)[:, :t].permute(0, 2, 1, 3).float()  # noqa: E731
    key = torch.arange(t, device="cuda")
    k, v = gather(s["k_pages"]), gather(s["v_pages"])
    v = torch.where((key < s["kv_len"][:, None])[:, None, :, None], v, 0.0)
    q = torch.zeros(b, n, hk, g, d, device="cuda")
    q[s["seq"], s["row"]] = s["q"].float().reshape(-1, hk, g, d)
    scores = (q.permute(0, 2, 3, 1, 4).reshape(b, hk, g * n, d) @ k.transpose(2, 3)).view(b, hk, g, n, t) / math.sqrt(d)
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
    seen = (seen & (at >= 0)[..., None])[:, None, None]
    top = torch.where(seen, scores, -math.inf).amax(-1, keepdim=True)
    w = torch.where(seen, (scores - top).exp(), 0.0)
    o = (w.view(b, hk, g * n, t) @ v).view(b, hk, g, n, d) / w.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4)[s["seq"], s["row"]].reshape(-1, hk * g, d).to(s["q"].dtype)


# ---------------------------------------------------------------- what an operator cannot do without, and its results in 64 bits
def work(case):
    size, d = 4 if case["dtype"] == "fp32" else 2, case["head_dim"]
    if case["kind"] == "attention":
        n, _ = _lengths(case)
        pairs, keys = _visible(case)
        return {"bytes": 2 * keys * case["kv_heads"] * d * size + 2 * sum(n) * case["heads"] * d * size, "flops": 4 * d * case["heads"] * pairs}
    moved = case["heads"] + case["kv_heads"] * (2 if case["kind"] == "append" else 1)
    tokens = case["tokens"] if case["kind"] == "norm_rope" else sum(_lengths(case)[0])
    return {"bytes": 2 * tokens * moved * d * size + 4 * tokens,
            "flops": tokens * (case["heads"] + case["kv_heads"]) * (3 * case["rotary"] + (4 * d if case["norm"] else 0))}


def exact(case, seed):
    s = prepare(case, seed)
    d = case["head_dim"]
    if case["kind"] == "attention":
        n, kv = _lengths(case)
        out, at, group = torch.zeros(sum(n), case["heads"], d, dtype=torch.float64, device="cuda"), 0, case["heads"] // case["kv_heads"]
        anc = _anc_of(case, n) if case["mask"] == "tree" else None
        for b, (m, t) in enumerate(zip(n, kv)):
            pages = s["table"][b, :-(-t // case["page"])].long()
            i, j = torch.arange(t - m, t, device="cuda")[:, None], torch.arange(t, device="cuda")[None]
            hidden = j > i
            if case["window"]:
                hidden = hidden | (i - j >= case["window"])
            if anc:
                rows = torch.tensor([[bool((words[c // 64] >> (c % 64)) & 1) for c in range(m)] for words in anc[b][0]], device="cuda")
                hidden = torch.cat([torch.zeros(m, t - m, dtype=torch.bool, device="cuda"), ~rows], 1)
            for h in range(case["kv_heads"]):
                take = lambda x: (x[pages, h] if case["order"] == "head" else x[pages, :, h]).reshape(-1, d)[:t].double()  # noqa: B023, E731
                k, v = take(s["k_pages"]), take(s["v_pages"])
                for e in range(h * group, (h + 1) * group):
                    logits = torch.einsum("id,jd->ij", s["q"][at:at + m, e].double(), k).mul_(d ** -0.5)
                    out[at:at + m, e] = torch.softmax(logits.masked_fill_(hidden, -math.inf), -1) @ v
            at += m
        return out
    turned = {}
    for name in ("q", "k"):
        x, gain = s[name].double(), s[name + "_gain"]
        if gain is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gain.double()
        p = (s["positions"] if case["kind"] == "norm_rope" else s["position"]).double()
        r = case["rotary"]
        pairs = torch.stack([x[..., 0:r:2], x[..., 1:r:2]], -1) if case["interleaved"] else torch.stack([x[..., :r // 2], x[..., r // 2:r]], -1)
        phase = torch.polar(torch.full((p.numel(), r // 2), _amplitude(case), dtype=torch.float64, device="cuda"),
                            p[:, None] * torch.tensor(_exact_frequencies(case), dtype=torch.float64, device="cuda"))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * phase[:, None])
        rotated = z.flatten(-2) if case["interleaved"] else torch.cat([z[..., 0], z[..., 1]], -1)
        turned[name] = torch.cat([rotated, x[..., r:]], -1)
    if case["kind"] == "norm_rope":
        return turned["q"], turned["k"]
    pages = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
    n, kv = _lengths(case)
    at = 0
    for b, (m, t) in enumerate(zip(n, kv)):
        where = torch.arange(t - m, t, device="cuda")
        page, slot = s["table"][b][where // case["page"]].long(), where % case["page"]
        for name, x in (("k", turned["k"]), ("v", s["v"].double())):
            view = pages[name] if case["order"] == "token" else pages[name].transpose(1, 2)
            view[page, slot] = x[at:at + m]
        at += m
    return turned["q"], pages["k"], pages["v"]


def _exact_frequencies(case):
    r, found = case["rotary"], []
    for i in range(r // 2):
        base = case["base"] * (case["factor"] ** (r / (r - 2)) if case["scaling"] == "base" else 1.0)
        f = math.exp(-2.0 * i / r * math.log(base))
        if case["scaling"] == "linear":
            f /= case["factor"]
        elif case["scaling"] == "rotations":
            turns = ORIGINAL / (2 * math.pi / f)
            f = f / case["factor"] if turns < 1 else f if turns > 4 else f * ((turns - 1) / 3 + (4 - turns) / 3 / case["factor"])
        elif case["scaling"] == "index":
            edge = [r * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (32.0, 1.0)]
            lo, hi = max(math.floor(edge[0]), 0), min(math.ceil(edge[1]), r - 1)
            slow = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = f * (slow / case["factor"] + 1 - slow)
        found.append(f)
    return found
