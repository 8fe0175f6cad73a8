"""What is measured of a decode step with drafted tokens: norms of queries and keys with rotary positions and the cache
write, attention of a tree of drafted tokens over a paged cache, sampling from the logits, and taking the drafted tokens
that the samples agree with into the cache.

`own` is set from outside: false, `run` is the operator written out in elementary torch operations; true, it is the call
a user makes of this package.  Head counts, head sizes and vocabularies are those of the LLaMA-3.2 1B / 3B / 11B / 90B
shapes in inputs/synth.py.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}
EPS = 1e-5
VOCAB = 128256


# ------------------------------------------------------------------------------------------ cases
def listed():
    heads, tree, sample, accept = ({"op": k} for k in ("heads", "tree", "sample", "accept"))
    return [
        # the drafted tokens of 4 sequences of the 3B model on their way into attention
        dict(heads, name="heads: 4 x 8 drafted", tokens=32, heads=24, kv_heads=8, dim=128, axes=1, interleaved=False, x="f32", page=16),
        # a prompt with image positions (time, height, width), 90B heads, odd length
        dict(heads, name="heads: prompt, 3 axes", tokens=2047, heads=64, kv_heads=8, dim=128, axes=3, interleaved=True, x="bf16", page=32),
        # a short chat on the 1B model that drafts 8 tokens: latency
        dict(tree, name="tree: one short", batch=1, longest=197, new=8, chain=False, heads=32, kv_heads=8, dim=64, page=16, lens=0),
        # a small serving batch of the 3B model, up to 16 drafted tokens each, lengths from a few tokens up
        dict(tree, name="tree: 8 ragged", batch=8, longest=8191, new=16, chain=False, heads=24, kv_heads=8, dim=128, page=16, lens=1),
        # one very long context with a wide tree, 11B heads: the split over the cache's length
        dict(tree, name="tree: one long", batch=1, longest=131071, new=31, chain=False, heads=32, kv_heads=8, dim=128, page=64, lens=0),
        # a full serving batch that drafts in a chain, 90B heads
        dict(tree, name="tree: 64 chains", batch=64, longest=16384, new=5, chain=True, heads=64, kv_heads=8, dim=128, page=32, lens=2),
        # the next pieces of two long prompts
        dict(tree, name="tree: prompt pieces", batch=2, longest=9001, new=1024, chain=True, heads=32, kv_heads=8, dim=128, page=32, lens=3),
        # the next token of one sequence, the usual settings
        dict(sample, name="sample: one token", rows=1, vocab=VOCAB, x="f32", set="k"),
        # a serving batch in which every sequence has settings of its own
        dict(sample, name="sample: 64 settings", rows=64, vocab=VOCAB, x="f32", set="all"),
        # every drafted token of 64 sequences, top-p alone
        dict(sample, name="sample: 64 x 8 drafted", rows=512, vocab=VOCAB, x="f32", set="p"),
        # one sequence of the 1B model, 16 layers
        dict(accept, name="accept: one sequence", batch=1, new=32, layers=16, kv_heads=8, dim=64, page=16, lens=0),
        # a serving batch of the 1B model with wide trees
        dict(accept, name="accept: 64 sequences", batch=64, new=48, layers=16, kv_heads=8, dim=64, page=32, lens=1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["heads", "tree", "tree", "sample", "sample", "accept"])
    heads, kv_heads, dim = rng.choice([(32, 8, 64), (24, 8, 128), (32, 8, 128), (64, 8, 128)])
    page = rng.choice([16, 24, 32, 64])
    if op == "heads":
        return {"op": op, "tokens": _log(rng, 1, 4096), "heads": heads, "kv_heads": kv_heads, "dim": dim, "axes": rng.choice([1, 3]),
                "interleaved": rng.choice([False, True]), "x": rng.choice(["bf16", "f32"]), "page": page}
    if op == "tree":
        batch = _log(rng, 1, 64)
        chain = rng.random() < 0.4
        new = _log(rng, 1, 1024 if chain else 64)
        longest = max(new, _log(rng, 1, min(131072, 64 * 16384 // batch)))
        while batch > 1 and batch * longest * new * heads > 64 * 16384 * 5 * 64:
            batch -= 1
        if batch * longest * new * heads > 2 * 64 * 16384 * 5 * 64:
            new = 5
        return {"op": op, "batch": batch, "longest": longest, "new": new, "chain": chain, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "page": page, "lens": rng.randrange(1, 1000)}
    if op == "sample":
        vocab = rng.choice([1024, 32000, 50257, VOCAB, VOCAB, VOCAB, _log(rng, 1, VOCAB)])
        return {"op": op, "rows": _log(rng, 1, 512), "vocab": vocab, "x": rng.choice(["f32", "f32", "bf16"]),
                "set": rng.choice(["k", "p", "all", "plain", "greedy", "min"])}
    return {"op": op, "batch": _log(rng, 1, 64), "new": _log(rng, 1, 64), "layers": rng.choice([1, 4, 16]), "kv_heads": kv_heads, "dim": 64 if dim == 64 else 128,
            "page": page, "lens": rng.randrange(1, 1000)}


def _shape(case):
    """(new tokens, states in the cache with them) of each sequence: the longest one first, the others spread over the range."""
    rng = random.Random(case["lens"])
    longest = case.get("longest", 40 + case["new"])
    out = [(case["new"], longest)]
    for _ in range(case["batch"] - 1):
        n = rng.randint(max(1, (case["new"] + 1) // 2), case["new"])
        out.append((n, rng.randint(n, longest)))
    return out


# ------------------------------------------------------------------------------------------ inputs
def _sections(case):
    pairs = case["dim"] // 2
    return [pairs] if case["axes"] == 1 else [pairs // 4, 3 * pairs // 8, 3 * pairs // 8]


def _table(n, dim):
    """cos | sin of position x frequency, [n][dim], as a model keeps it (base 500000)."""
    f = 500000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _page_table(lens, page, g):
    """Pages of each sequence, scattered over the pool; entries past a sequence's pages are 0."""
    need = [-(-n // page) for n in lens]
    pool = sum(need) + 3
    perm = torch.randperm(pool, generator=g, device="cuda", dtype=torch.int64)
    table = torch.zeros(len(lens), max(need), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n].int()
        at += n
    return table, pool


def _parents(n, rng, chain=False):
    """A tree of n tokens in the order they were drafted: token 0 is the last one that is certain, a parent comes before its children."""
    return [-1] + [i - 1 if chain else rng.randrange(max(0, i - 9), i) for i in range(1, n)]


def _ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)

    def randn(*shape, dtype=torch.float32, scale=1.0):
        x = torch.randn(*shape, generator=g, device="cuda", dtype=dtype)
        return x if scale == 1.0 else x.mul_(scale)

    s = {"case": dict(case)}
    if case["op"] == "heads":
        T, H, K, D, page = (case[k] for k in ("tokens", "heads", "kv_heads", "dim", "page"))
        dt = DTYPES[case["x"]]
        s["q"], s["k"], s["v"] = (randn(T, n, D, dtype=dt, scale=2.0) for n in (H, K, K))
        s["q_weight"], s["k_weight"] = (randn(D, scale=0.2).add_(1.0) for _ in range(2))
        i = torch.arange(T, device="cuda")
        if case["axes"] == 3:
            pos = torch.stack([i // 64, (i // 8) % 8, i % 8])
        else:
            pos = (i if T > 64 else torch.randint(0, 8192, (T,), generator=g, device="cuda"))[None]
        s["positions"] = pos.int().contiguous()
        s["table"] = _table(8192, D)
        s["sections"] = _sections(case)
        s["axis"] = torch.tensor([axis for axis, n in enumerate(s["sections"]) for _ in range(n)], device="cuda")
        # tokens fill pages in order; the last sixteenth of them is padding of the batch and has no slot
        pages = -(-T // page) + 1
        perm = torch.randperm(pages, generator=g, device="cuda")
        slots = perm[i // page] * page + i % page
        s["written"] = T - T // 16
        slots[s["written"]:] = -1
        s["slots"] = slots.int()
        s["k_pool"], s["v_pool"] = (randn(pages, K, page, D, dtype=torch.bfloat16) for _ in range(2))
    elif case["op"] == "tree":
        H, K, D, page = (case[k] for k in ("heads", "kv_heads", "dim", "page"))
        shape = _shape(case)
        s["page_table"], pool = _page_table([n for _, n in shape], page, g)
        s["lens"] = _ints([n for _, n in shape])
        firsts = [0]
        for n, _ in shape:
            firsts.append(firsts[-1] + n)
        s["first"], s["firsts"] = _ints(firsts), firsts
        s["mask"], s["seen"] = None, None
        if not case["chain"]:  # bit j of a token's words: it sees the sequence's new token j (itself and the tokens it follows)
            words = -(-case["new"] // 32)
            rows = []
            for n, _ in shape:
                sees = []
                for i, parent in enumerate(_parents(n, rng)):
                    sees.append((sees[parent] if i else 0) | 1 << i)
                rows += sees
            s["mask"] = _ints([[(r >> 32 * w & 0xFFFFFFFF) - ((r >> 32 * w + 31 & 1) << 32) for w in range(words)] for r in rows])
        s["q"] = randn(firsts[-1], H, D, dtype=torch.bfloat16, scale=1.5)
        s["k_pool"], s["v_pool"] = (randn(pool, K, page, D, dtype=torch.bfloat16) for _ in range(2))
    elif case["op"] == "sample":
        R, V, kind = case["rows"], case["vocab"], case["set"]
        # a broad floor and, in other tokens for every row, a head that falls off with the rank; a third of the rows have hardly more than
        # the floor, the others are the sharper the higher their head; a few tokens are never allowed
        x = randn(R, V, scale=1.5)
        n = min(V, 256)
        at = torch.randint(0, V, (R, n), generator=g, device="cuda")
        sharp = torch.rand(R, 1, generator=g, device="cuda")
        x.scatter_add_(1, at, (9.0 + 11.0 * sharp) - (1.0 + sharp) * torch.arange(1, n + 1, device="cuda").log()[None])
        if V > 8:
            x[:, 3] = x[:, 5] = -math.inf
        s["logits"] = x.to(DTYPES[case["x"]])
        s["uniform"] = torch.rand(R, generator=g, device="cuda")

        def each(*choices):
            return [rng.choice(choices) for _ in range(R)]

        s["temperature"] = s["top_k"] = s["top_p"] = s["min_p"] = None
        if kind == "greedy":
            s["temperature"] = _ints([0.0] * R, torch.float32)
        elif kind != "plain":
            s["temperature"] = _ints(each(0.6, 0.7, 0.8, 1.0) if kind != "all" else each(0.0, 0.3, 0.7, 1.0, 1.5), torch.float32)
        if kind in ("k", "all"):
            s["top_k"] = _ints([50] * R if kind == "k" else each(0, 0, 1, 20, 50, 1000))
        if kind in ("k", "p", "all"):
            s["top_p"] = _ints(each(0.9, 0.95) if kind != "all" else each(0.5, 0.9, 0.99, 1.0), torch.float32)
        if kind in ("min", "all"):
            s["min_p"] = _ints(each(0.05, 0.1) if kind == "min" else each(0.0, 0.0, 0.02, 0.1), torch.float32)
    else:
        K, D, page, layers = (case[k] for k in ("kv_heads", "dim", "page", "layers"))
        shape = _shape(case)
        s["page_table"], pool = _page_table([n for _, n in shape], page, g)
        s["lens"] = _ints([n for _, n in shape])
        firsts, parents, tokens, sampled = [0], [], [], []
        for n, _ in shape:
            firsts.append(firsts[-1] + n)
            mine = _parents(n, rng)
            drafted = [rng.randrange(VOCAB) for _ in range(n)]
            drawn = [rng.randrange(VOCAB) for _ in range(n)]
            # a path that the samples agree with; its tokens lie past the slots they move to, so that a pass can be repeated
            leaf = rng.randrange(n)
            path = [leaf]
            while path[0]:
                path.insert(0, mine[path[0]])
            while any(0 < c < len(path) for c in path):
                path.pop()
            for a, b in zip(path, path[1:]):
                drawn[a] = drafted[b]
            parents += mine
            tokens += drafted
            sampled += drawn
        s["first"], s["firsts"] = _ints(firsts), firsts
        s["parents"], s["tokens"], s["sampled"] = _ints(parents), _ints(tokens), _ints(sampled)
        s["max_path"] = 16
        s["k_pool"], s["v_pool"] = (randn(layers, pool, K, page, D, dtype=torch.bfloat16) for _ in range(2))
    if own:
        from paper_2509_22951_b200 import binding as tq

        s["tq"] = tq
        if case["op"] == "accept":
            s["caches"] = tq.tq_kv_caches([tq.tq_kv_cache(k, v) for k, v in zip(s["k_pool"], s["v_pool"])])
        elif "k_pool" in s:
            s["cache"] = tq.tq_kv_cache(s["k_pool"], s["v_pool"])
        if case["op"] == "tree":
            s["workspace"] = tq.tq_attn_workspace()
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _plain_heads(s):
    case = s["case"]
    pairs, n, page = case["dim"] // 2, s["written"], case["page"]
    pos, pair = s["positions"].long()[s["axis"]].t(), torch.arange(pairs, device="cuda")  # each pair goes by the axis of its section
    cos, sin = s["table"][pos, pair][:, None], s["table"][pos, pairs + pair][:, None]

    def turned(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        if case["interleaved"]:
            a, b = x[..., 0::2], x[..., 1::2]
            return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2).to(torch.bfloat16)
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1).to(torch.bfloat16)

    q, k = turned(s["q"], s["q_weight"]), turned(s["k"], s["k_weight"])
    slots = s["slots"][:n].long()
    s["k_pool"][slots // page, :, slots % page] = k[:n]
    s["v_pool"][slots // page, :, slots % page] = s["v"][:n].to(torch.bfloat16)
    return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _own_heads(s):
    q = s["tq"].tq_qk_norm_rope_append(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["table"], s["positions"], s["slots"], s["cache"],
                                       eps=EPS, sections=s["sections"], interleaved=s["case"]["interleaved"])
    return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _plain_tree(s):
    case = s["case"]
    H, K, D, page = (case[k] for k in ("heads", "kv_heads", "dim", "page"))
    out = torch.empty_like(s["q"])
    for b, (n, length) in enumerate(_shape(case)):
        rows = slice(s["firsts"][b], s["firsts"][b + 1])
        pages = s["page_table"][b, :-(-length // page)].long()
        k, v = (s[x][pages].transpose(0, 1).flatten(1, 2)[:, :length].float() for x in ("k_pool", "v_pool"))  # [K][length][D]
        at, state = torch.arange(n, device="cuda")[:, None], torch.arange(length, device="cuda")[None] - (length - n)
        if s["mask"] is None:
            seen = state <= at
        else:
            j = state.clamp(min=0).expand(n, -1)
            seen = (state < 0) | ((s["mask"][rows].gather(1, j // 32) >> (j % 32)) & 1 != 0)
        q = s["q"][rows].float().view(n, K, H // K, D).permute(1, 2, 0, 3)  # [K][group][n][D]
        x = (q @ k[:, None].transpose(-1, -2)) * (1.0 / math.sqrt(D))
        x = x.masked_fill(~seen, float("-inf"))
        p = torch.exp(x - x.amax(-1, keepdim=True))
        o = (p @ v[:, None]) / p.sum(-1, keepdim=True)
        out[rows] = o.permute(2, 0, 1, 3).reshape(n, H, D).to(torch.bfloat16)
    return out


def _own_tree(s):
    return s["tq"].tq_tree_attention(s["q"], s["cache"], s["page_table"], s["first"], s["lens"], s["workspace"], mask=s["mask"])


def _plain_sample(s):
    x = s["logits"].double()
    R, V = x.shape
    rank = torch.arange(V, device="cuda")
    top = x.amax(-1, keepdim=True)
    best = torch.where(x == top, rank, V).amin(-1)
    t = torch.ones(R, device="cuda") if s["temperature"] is None else s["temperature"]
    w = torch.exp((x - top) / torch.where(t > 0, t, 1.0).double()[:, None])
    w_sorted, token = w.sort(dim=-1, descending=True, stable=True)
    keep = torch.ones(R, V, dtype=torch.bool, device="cuda")
    if s["top_k"] is not None:
        keep &= (rank < s["top_k"][:, None]) | (s["top_k"] <= 0)[:, None]
    if s["top_p"] is not None:
        kept = w_sorted * keep
        upto = kept.cumsum(-1)
        keep &= upto - kept < s["top_p"].double()[:, None] * upto[:, -1:]
    if s["min_p"] is not None:
        keep &= w_sorted >= s["min_p"].double()[:, None]
    w = torch.zeros_like(w).scatter_(1, token, w_sorted * keep)
    upto = w.cumsum(-1)
    total = upto[:, -1]
    drawn = (upto <= s["uniform"].double()[:, None] * total[:, None]).sum(-1).clamp(max=V - 1)
    drawn = torch.where(t > 0, drawn, best)
    logprob = torch.where(t > 0, torch.log(w.gather(1, drawn[:, None])[:, 0] / total), 0.0)
    return {"token": drawn.int(), "logprob": logprob.float()}


def _own_sample(s):
    token, logprob = s["tq"].tq_sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                       min_p=s["min_p"], logprob=True)
    return {"token": token, "logprob": logprob}


def _plain_accept(s):
    case = s["case"]
    B, page, deepest = case["batch"], case["page"], s["max_path"]
    first, new = s["first"][:-1].long(), s["first"].diff().long()
    context = s["lens"].long() - new
    i = torch.arange(case["new"], device="cuda")[None]
    there = i < new[:, None]
    rows = (first[:, None] + i).clamp(max=s["tokens"].numel() - 1)
    parents, tokens, sampled = (s[x][rows] for x in ("parents", "tokens", "sampled"))
    path = torch.full((B, deepest), -1, dtype=torch.int32, device="cuda")
    out = torch.full((B, deepest), -1, dtype=torch.int32, device="cuda")
    at, going = torch.zeros(B, dtype=torch.int64, device="cuda"), torch.ones(B, dtype=torch.bool, device="cuda")
    for d in range(deepest):
        drawn = sampled.gather(1, at[:, None])[:, 0]
        path[:, d] = torch.where(going, at, -1)
        out[:, d] = torch.where(going, drawn, -1)
        follows = there & (parents == at[:, None]) & (tokens == drawn[:, None])
        child = torch.where(follows, i, case["new"]).amin(1)
        going = going & (child < new)
        at = torch.where(going, child, at)
    count = (path >= 0).sum(1).int()
    d = torch.arange(deepest, device="cuda")[None]
    moved = path >= 0

    def places(x):  # page and slot of the states that path entries are in, or go to
        x = (context[:, None] + x)[moved]
        b = torch.arange(B, device="cuda")[:, None].expand(-1, deepest)[moved]
        return s["page_table"][b, x // page].long(), x % page

    (p0, s0), (p1, s1) = places(path.long()), places(d.expand(B, -1))
    for pool in (s["k_pool"], s["v_pool"]):
        pool[:, p1, :, s1] = pool[:, p0, :, s0]
    return {"tokens": out, "path": path, "count": count, "lens": (context + count).int(), "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _own_accept(s):
    tokens, path, count, lens = s["tq"].tq_tree_accept(s["caches"], s["page_table"], s["first"], s["lens"], s["tokens"], s["parents"], s["sampled"],
                                                       max_path=s["max_path"])
    return {"tokens": tokens, "path": path, "count": count, "lens": lens, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


_plain = {"heads": _plain_heads, "tree": _plain_tree, "sample": _plain_sample, "accept": _plain_accept}
_own = {"heads": _own_heads, "tree": _own_tree, "sample": _own_sample, "accept": _own_accept}


# ------------------------------------------------------------------------------------------ floors
def work(case):
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * SIZES[case["x"]] + 28 * case["rows"], "flops": 8 * n}
    K, D = case["kv_heads"], case["dim"]
    if case["op"] == "heads":
        T, H = case["tokens"], case["heads"]
        kept = T - T // 16  # tokens with a slot: the others' keys and values need not be read
        read = (T * H + 2 * kept * K) * D * SIZES[case["x"]] + 4 * D * T + 4 * T * (case["axes"] + 1) + 8 * D
        return {"bytes": read + (T * H + 2 * kept * K) * D * 2, "flops": 8 * (T * H + kept * K) * D}
    shape = _shape(case)
    tokens, states = sum(n for n, _ in shape), sum(n for _, n in shape)
    if case["op"] == "tree":
        H = case["heads"]
        # a token sees the context and, of the new tokens, those it follows: half of them in a chain, few in a tree
        pairs = sum(n * (length - n) + (n * (n + 1) // 2 if case["chain"] else n) for n, length in shape)
        mask = 0 if case["chain"] else 4 * tokens * -(-case["new"] // 32)
        return {"bytes": 4 * states * K * D + 4 * tokens * H * D + 4 * -(-states // case["page"]) + 8 * case["batch"] + mask, "flops": 4 * pairs * H * D}
    # the walk's inputs and outputs, and one token of a sequence, about, that moves in every layer
    moved = case["batch"] * case["layers"] * 2 * K * D * 2 * 2
    return {"bytes": moved + 12 * tokens + (8 + 2 * 4 * 16 + 8) * case["batch"], "flops": tokens}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "heads":
        T, D, page = (case[k] for k in ("tokens", "dim", "page"))
        pairs, angle, at = D // 2, [], 0
        for axis, n in enumerate(s["sections"]):
            f = 500000.0 ** (-torch.arange(at, at + n, dtype=f64, device="cuda") / pairs)
            angle.append(s["positions"][axis].to(f64)[:, None] * f)
            at += n
        turn = torch.polar(torch.ones(T, 1, pairs, dtype=f64, device="cuda"), torch.cat(angle, 1)[:, None])

        def rotated(x, w):
            x = x.to(f64)
            x = x / torch.sqrt(torch.mean(x ** 2, dim=-1) + EPS)[..., None] * w.to(f64)
            z = torch.view_as_complex(x.view(T, -1, pairs, 2) if case["interleaved"] else
                                      x.view(T, -1, 2, pairs).transpose(2, 3).contiguous()) * turn
            z = torch.view_as_real(z)
            return (z if case["interleaved"] else z.transpose(2, 3)).reshape(x.shape)

        out = {"q": rotated(s["q"], s["q_weight"]), "k_pool": s["k_pool"].to(f64), "v_pool": s["v_pool"].to(f64)}
        n = s["written"]
        at = s["slots"][:n].long()
        for name, x in (("k_pool", rotated(s["k"], s["k_weight"])), ("v_pool", s["v"].to(f64))):
            flat = out[name].transpose(1, 2).reshape(-1, case["kv_heads"], D)  # [slot][head][D]
            flat[at] = x[:n]
            out[name] = flat.view(-1, page, case["kv_heads"], D).transpose(1, 2)
        return out
    if case["op"] == "tree":
        H, K, D, page = (case[k] for k in ("heads", "kv_heads", "dim", "page"))
        G = H // K
        out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
        for b, (n, length) in enumerate(_shape(case)):
            at, context = s["firsts"][b], length - n
            pages = s["page_table"][b, :-(-length // page)].long()
            hidden = torch.zeros(n, length, dtype=torch.bool, device="cuda")
            for j in range(n):
                sees = torch.arange(n, device="cuda") >= j if s["mask"] is None else (s["mask"][at:at + n, j // 32].long() >> j % 32) % 2 == 1
                hidden[:, context + j] = ~sees
            for h in range(K):
                k, v = (s[x][pages, h].reshape(-1, D)[:length].to(f64) for x in ("k_pool", "v_pool"))
                for i in range(h * G, (h + 1) * G):
                    x = s["q"][at:at + n, i].to(f64) @ k.T / D ** 0.5
                    out[at:at + n, i] = torch.softmax(x.masked_fill_(hidden, -math.inf), dim=1) @ v
        return out
    if case["op"] == "sample":
        R, V = case["rows"], case["vocab"]
        token, logprob = torch.zeros(R, dtype=torch.int32), torch.zeros(R, dtype=f64)
        setting = {k: None if s[k] is None else s[k].tolist() for k in ("uniform", "temperature", "top_k", "top_p", "min_p")}
        x = s["logits"].to(f64)
        value, place = x.sort(dim=1, descending=True, stable=True)
        for r in range(R):
            T = 1.0 if setting["temperature"] is None else setting["temperature"][r]
            if T <= 0.0:
                token[r] = int(place[r, 0])
                continue
            n = V
            if setting["top_k"] is not None and 0 < setting["top_k"][r] < V:
                n = setting["top_k"][r]
            mass = torch.softmax(value[r, :n] / T, 0)
            if setting["top_p"] is not None and setting["top_p"][r] < 1.0:
                before = torch.cat([mass.new_zeros(1), mass.cumsum(0)[:-1]])
                mass = mass[before < setting["top_p"][r]]
            if setting["min_p"] is not None:
                mass = mass[mass >= setting["min_p"][r] * mass[0]]
            ids, order = place[r, :mass.numel()].sort()
            mass = mass[order] / mass.sum()
            at = int(torch.searchsorted(mass.cumsum(0), torch.tensor(setting["uniform"][r], dtype=f64, device="cuda"), right=True))
            at = min(at, ids.numel() - 1)
            token[r], logprob[r] = int(ids[at]), float(mass[at].log())
        return {"token": token.cuda(), "logprob": logprob.cuda()}
    K, D, page = (case[k] for k in ("kv_heads", "dim", "page"))
    paths, drawn, parents, tokens, sampled = [], [], *(s[x].tolist() for x in ("parents", "tokens", "sampled"))
    pools = {x: s[x].clone() for x in ("k_pool", "v_pool")}
    lens, table = [], s["page_table"].tolist()
    source, target = [], []
    for b, (n, length) in enumerate(_shape(case)):
        f, path = s["firsts"][b], [0]
        while len(path) < s["max_path"]:
            after = [c for c in range(n) if parents[f + c] == path[-1] and tokens[f + c] == sampled[f + path[-1]]]
            if not after:
                break
            path.append(after[0])
        fill = [-1] * (s["max_path"] - len(path))
        paths.append(path + fill)
        drawn.append([sampled[f + c] for c in path] + fill)
        lens.append(length - n + len(path))
        for d, c in enumerate(path):
            for x, at in ((length - n + c, source), (length - n + d, target)):
                at.append(table[b][x // page] * page + x % page)
    for x in pools:
        flat = pools[x].transpose(2, 3).reshape(case["layers"], -1, K, D)
        flat[:, target] = flat[:, source]
        pools[x] = flat.view(case["layers"], -1, page, K, D).transpose(2, 3)
    return {"tokens": _ints(drawn), "path": _ints(paths), "count": _ints([sum(c >= 0 for c in p) for p in paths]), "lens": _ints(lens), **pools}
