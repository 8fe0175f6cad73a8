"""What is measured of the operators between a decoder's linear layers: normalisation, rotary positions
with the cache write, attention of one new token over a paged cache, attention to an encoder's states.

`own` is set from outside: false, `run` is the operator written out in elementary torch operations in 32
bits; true, it is the call a user makes of this package.  Head counts, head sizes and hidden sizes are those
of the LLaMA-3.2 1B / 3B / 11B / 90B shapes in inputs/synth.py; 6404 encoder states are four image tiles
of 1601 patches.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}
EPS = 1e-5
TILE = 1601  # encoder states of one image tile


# ------------------------------------------------------------------------------------------ cases
def listed():
    norm, rope, paged, cross = ({"op": k} for k in ("norm", "rope", "paged", "cross"))
    return [
        # one token of the 1B model on its way into a layer: bf16 stream, fp32 output of the product before
        dict(norm, name="norm: one token", rows=1, cols=2048, h="bf16", delta="f32", out="bf16"),
        # a prompt through the 90B model's norm, fp32 stream
        dict(norm, name="norm: prompt", rows=2049, cols=8192, h="f32", delta="f32", out="bf16"),
        # a prompt's activations to 8 bits with a scale for each row
        dict(norm, name="norm: prompt to 8 bits", rows=1023, cols=4096, h="bf16", delta="bf16", out="q8"),
        # the norm of every key head of an image's encoder states
        dict(norm, name="norm: heads", rows=8 * 6404, cols=128, h="bf16", delta="", out="bf16"),
        # one decode step of 8 sequences of the 3B model
        dict(rope, name="rope: 8 tokens", tokens=8, heads=24, kv_heads=8, dim=128, axes=1, interleaved=False, x="f32", page=16),
        # a prompt with image positions (time, height, width), 11B heads, odd length
        dict(rope, name="rope: prompt, 3 axes", tokens=2047, heads=32, kv_heads=8, dim=128, axes=3, interleaved=True, x="f32", page=32),
        # a short chat on the 1B model: latency
        dict(paged, name="paged: one short", batch=1, longest=37, heads=32, kv_heads=8, dim=64, page=16, lens=0),
        # a small serving batch of the 3B model, lengths from a few tokens up
        dict(paged, name="paged: 8 ragged", batch=8, longest=8191, heads=24, kv_heads=8, dim=128, page=16, lens=1),
        # one very long context, 11B heads: the split over the cache's length
        dict(paged, name="paged: one long", batch=1, longest=131071, heads=32, kv_heads=8, dim=128, page=64, lens=0),
        # a full serving batch, 90B heads
        dict(paged, name="paged: 64 ragged", batch=64, longest=16384, heads=64, kv_heads=8, dim=128, page=32, lens=2),
        # one new token of 4 sequences that look at an image of up to four tiles
        dict(cross, name="cross: one token", batch=4, tokens=1, states=4 * TILE, heads=32, kv_heads=8, dim=128, tiles=4, first=0),
        # prompts of 2 sequences, 90B heads; the text before the image sees none of its states
        dict(cross, name="cross: prompt", batch=2, tokens=2048, states=4 * TILE, heads=64, kv_heads=8, dim=128, tiles=4, first=33),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "rope", "paged", "cross"])
    heads, kv_heads, dim = rng.choice([(32, 8, 64), (24, 8, 128), (32, 8, 128), (64, 8, 128)])
    if op == "norm":
        cols = rng.choice([64, 128, 1000, 2047, 2048, 3072, 4096, 5001, 8192])
        rows = _log(rng, 1, min(65536, 2049 * 8192 // cols))
        out = rng.choice(["bf16", "bf16", "q8"])
        return {"op": op, "rows": rows, "cols": cols, "h": rng.choice(["bf16", "f32"]), "delta": rng.choice(["", "bf16", "f32"]), "out": out}
    if op == "rope":
        return {"op": op, "tokens": _log(rng, 1, 4096), "heads": heads, "kv_heads": kv_heads, "dim": dim, "axes": rng.choice([1, 3]),
                "interleaved": rng.choice([False, True]), "x": rng.choice(["bf16", "f32"]), "page": rng.choice([16, 24, 32, 64])}
    if op == "paged":
        batch = _log(rng, 1, 64)
        longest = _log(rng, 1, min(131072, 64 * 16384 // batch))
        return {"op": op, "batch": batch, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim,
                "page": rng.choice([16, 24, 32, 64]), "lens": rng.randrange(1, 1000)}
    batch = rng.choice([1, 2, 3, 4])
    tokens = rng.choice([1, _log(rng, 2, 2048), _log(rng, 2, 2048)])
    tiles = rng.choice([0, 1, 2, 4])
    states = TILE * tiles if tiles else _log(rng, 1, 4 * TILE)
    while batch * tokens * heads > 2 * 2048 * 64:
        batch -= 1
    return {"op": op, "batch": batch, "tokens": tokens, "states": states, "heads": heads, "kv_heads": kv_heads, "dim": dim, "tiles": tiles,
            "first": 0 if tokens == 1 else rng.randrange(0, min(tokens, 64))}


def _lengths(case):
    """Cached tokens of each sequence of a paged case: the longest one first, the others spread over the range."""
    rng = random.Random(case["lens"])
    return [case["longest"]] + [rng.randint(1, case["longest"]) for _ in range(case["batch"] - 1)]


def _cross_lens(case):
    """Valid encoder states of each sequence: all with image tiles (the mask says the rest), else padded to the longest."""
    if case["tiles"]:
        return [case["states"]] * case["batch"]
    return [max(1, case["states"] * (4 - b) // 4) for b in range(case["batch"])]


def _cross_tiles(case):
    """Image tiles that each sequence has."""
    return [max(1, case["tiles"] - b % 3) for b in range(case["batch"])] if case["tiles"] else []


# ------------------------------------------------------------------------------------------ inputs
def _sections(case):
    pairs = case["dim"] // 2
    return [pairs] if case["axes"] == 1 else [pairs // 4, 3 * pairs // 8, 3 * pairs // 8]


def _table(n, dim):
    """cos | sin of position x frequency, [n][dim], as a model keeps it (base 500000)."""
    f = 500000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _page_table(case, g):
    """Pages of each sequence, scattered over the pool; entries past a sequence's pages are 0."""
    lens, page = _lengths(case), case["page"]
    need = [-(-n // page) for n in lens]
    pool = sum(need) + 3
    perm = torch.randperm(pool, generator=g, device="cuda", dtype=torch.int64)
    table = torch.zeros(case["batch"], max(need), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n].int()
        at += n
    return table, pool


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape, dtype=torch.float32, scale=1.0):
        x = torch.randn(*shape, generator=g, device="cuda", dtype=dtype)
        return x if scale == 1.0 else x.mul_(scale)

    s = {"case": dict(case)}
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        s["h"] = randn(rows, cols, dtype=DTYPES[case["h"]], scale=3.0)
        s["delta"] = randn(rows, cols, dtype=DTYPES[case["delta"]]) if case["delta"] else None
        s["weight"] = randn(cols, scale=0.2).add_(1.0)
        s["h_out"] = torch.empty_like(s["h"]) if case["delta"] else None
    elif case["op"] == "rope":
        T, H, K, D, page = (case[k] for k in ("tokens", "heads", "kv_heads", "dim", "page"))
        dt = DTYPES[case["x"]]
        s["q"], s["k"], s["v"] = (randn(T, n, D, dtype=dt) for n in (H, K, K))
        i = torch.arange(T, device="cuda")
        if case["axes"] == 3:
            pos = torch.stack([i // 64, (i // 8) % 8, i % 8])
        else:
            pos = (i if T > 64 else torch.randint(0, 8192, (T,), generator=g, device="cuda"))[None]
        s["positions"] = pos.int().contiguous()
        s["table"] = _table(8192, D)
        s["sections"] = _sections(case)
        s["axis"] = torch.tensor([axis for axis, n in enumerate(s["sections"]) for _ in range(n)], device="cuda")
        # tokens of a prompt fill pages in order, those of a decode step lie in a page each; the last sixteenth of the
        # tokens is padding of the batch and has no slot
        pages = -(-T // page) + 1 if T > 64 else T + 1
        perm = torch.randperm(pages, generator=g, device="cuda")
        slots = perm[i // page] * page + i % page if T > 64 else perm[i] * page + i % page
        s["written"] = T - T // 16
        slots[s["written"]:] = -1
        s["slots"] = slots.int()
        s["k_pool"], s["v_pool"] = (randn(pages, K, page, D, dtype=torch.bfloat16) for _ in range(2))
    elif case["op"] == "paged":
        B, H, K, D, page = (case[k] for k in ("batch", "heads", "kv_heads", "dim", "page"))
        s["page_table"], pool = _page_table(case, g)
        s["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        s["q"] = randn(B, H, D, dtype=torch.bfloat16, scale=1.5)
        s["k_pool"], s["v_pool"] = (randn(pool, K, page, D, dtype=torch.bfloat16) for _ in range(2))
    else:
        B, T, S, H, K, D, n = (case[k] for k in ("batch", "tokens", "states", "heads", "kv_heads", "dim", "tiles"))
        s["q"] = randn(B, T, H, D, dtype=torch.bfloat16, scale=1.5)
        s["k"], s["v"] = (randn(B, S, K, D, dtype=torch.bfloat16) for _ in range(2))
        s["kv_len"] = torch.tensor(_cross_lens(case), dtype=torch.int32, device="cuda")
        s["mask"] = None
        if n:  # token t sees the tiles its sequence has once the image has been named
            has = torch.tensor(_cross_tiles(case), device="cuda")[:, None, None]
            t = torch.arange(T, device="cuda")[None, :, None]
            s["mask"] = ((torch.arange(n, device="cuda")[None, None] < has) & (t >= case["first"])).to(torch.uint8).contiguous()
    if own:
        from paper_2509_22951_b200 import binding as tq

        s["tq"] = tq
        if "k_pool" in s:
            s["cache"] = tq.tq_kv_cache(s["k_pool"], s["v_pool"])
        if case["op"] in ("paged", "cross"):
            s["workspace"] = tq.tq_attn_workspace()
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _plain_norm(s):
    case = s["case"]
    x = s["h"].float()
    if s["delta"] is not None:
        x = x + s["delta"].float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    out = {}
    if s["delta"] is not None:
        out["h"] = x.to(s["h"].dtype)
    if case["out"] == "bf16":
        out["out"] = y.to(torch.bfloat16)
        return out
    top = y.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, top / 127.0, torch.ones_like(top))
    out["values"] = (y / scale).round().clamp(-127, 127).to(torch.int8) * scale
    return out


def _own_norm(s):
    tq = s["tq"]
    out = {}
    if s["delta"] is not None:
        out["h"] = s["h_out"]
    if s["case"]["out"] == "bf16":
        out["out"] = tq.tq_rmsnorm(s["h"], s["weight"], s["delta"], eps=EPS, h_out=s["h_out"])
        return out
    q, scale = tq.tq_rmsnorm_q8(s["h"], s["weight"], s["delta"], eps=EPS, h_out=s["h_out"])
    out["values"] = q * scale[:, None]
    return out


def _angles(s):
    """cos and sin of every pair of every token, [T][1][pairs]: each pair goes by the axis of its section."""
    pairs = s["case"]["dim"] // 2
    pos = s["positions"].long()[s["axis"]].t()  # [T][pairs]
    pair = torch.arange(pairs, device="cuda")
    return s["table"][pos, pair][:, None], s["table"][pos, pairs + pair][:, None]


def _rotate(x, cos, sin, interleaved):
    x = x.float()
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _plain_rope(s):
    case = s["case"]
    cos, sin = _angles(s)
    n, page = s["written"], case["page"]
    q = _rotate(s["q"], cos, sin, case["interleaved"]).to(torch.bfloat16)
    k = _rotate(s["k"], cos, sin, case["interleaved"]).to(torch.bfloat16)
    slots = s["slots"][:n].long()
    s["k_pool"][slots // page, :, slots % page] = k[:n]
    s["v_pool"][slots // page, :, slots % page] = s["v"][:n].to(torch.bfloat16)
    return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _own_rope(s):
    q = s["tq"].tq_rope_append(s["q"], s["k"], s["v"], s["table"], s["positions"], s["slots"], s["cache"], sections=s["sections"],
                               interleaved=s["case"]["interleaved"])
    return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _attend(q, k, v, seen):
    """q [..., n, D], k / v [..., m, D], seen [..., n or 1, m]: a row that sees nothing gives zeros."""
    x = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(q.shape[-1]))
    x = x.masked_fill(~seen, float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top.isfinite(), top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    return (p @ v) / torch.where(total > 0, total, torch.ones_like(total))


def _plain_paged(s):
    case = s["case"]
    B, H, K, D = (case[k] for k in ("batch", "heads", "kv_heads", "dim"))
    table = s["page_table"].long()
    k, v = (s[n][table].transpose(1, 2).flatten(2, 3).float() for n in ("k_pool", "v_pool"))  # [B][K][length][D]
    seen = torch.arange(k.shape[2], device="cuda")[None] < s["lens"][:, None]
    out = _attend(s["q"].float().view(B, K, H // K, D), k, v, seen[:, None, None])
    return out.reshape(B, H, D).to(torch.bfloat16)


def _own_paged(s):
    return s["tq"].tq_paged_attention(s["q"], s["cache"], s["page_table"], s["lens"], s["workspace"])


def _plain_cross(s):
    case = s["case"]
    B, T, S, H, K, D = (case[k] for k in ("batch", "tokens", "states", "heads", "kv_heads", "dim"))
    seen = (torch.arange(S, device="cuda")[None] < s["kv_len"][:, None])[:, None]
    if s["mask"] is not None:
        seen = seen & s["mask"].bool().repeat_interleave(S // case["tiles"], -1, output_size=S)
    q = s["q"].float().view(B, T, K, H // K, D).permute(0, 2, 3, 1, 4)  # [B][K][group][T][D]
    k, v = (s[n].float().transpose(1, 2)[:, :, None] for n in ("k", "v"))
    out = _attend(q, k, v, seen[:, None, None])
    return out.permute(0, 3, 1, 2, 4).reshape(B, T, H, D).to(torch.bfloat16)


def _own_cross(s):
    case = s["case"]
    return s["tq"].tq_cross_attention(s["q"], s["k"], s["v"], s["workspace"], kv_len=s["kv_len"], mask=s["mask"],
                                      block_len=case["states"] // case["tiles"] if case["tiles"] else 0)


_plain = {"norm": _plain_norm, "rope": _plain_rope, "paged": _plain_paged, "cross": _plain_cross}
_own = {"norm": _own_norm, "rope": _own_rope, "paged": _own_paged, "cross": _own_cross}


# ------------------------------------------------------------------------------------------ floors
def work(case):
    if case["op"] == "norm":
        n, h = case["rows"] * case["cols"], SIZES[case["h"]]
        b = n * h + 4 * case["cols"] + n * (2 if case["out"] == "bf16" else 1)
        if case["delta"]:
            b += n * (SIZES[case["delta"]] + h)
        return {"bytes": b, "flops": 6 * n}
    if case["op"] == "rope":
        T, H, K, D = (case[k] for k in ("tokens", "heads", "kv_heads", "dim"))
        kept = T - T // 16  # tokens with a slot: the others' keys and values need not be read
        read = (T * H + 2 * kept * K) * D * SIZES[case["x"]] + 4 * D * T + 4 * T * (case["axes"] + 1)
        return {"bytes": read + (T * H + 2 * kept * K) * D * 2, "flops": 3 * (T * H + kept * K) * D}
    H, K, D = (case[k] for k in ("heads", "kv_heads", "dim"))
    if case["op"] == "paged":
        n = sum(_lengths(case))
        return {"bytes": 4 * n * K * D + 4 * case["batch"] * H * D + 4 * -(-n // case["page"]) + 4 * case["batch"], "flops": 4 * n * H * D}
    B, T = case["batch"], case["tokens"]
    if case["tiles"]:
        per = case["states"] // case["tiles"]
        seen = [n * per for n in _cross_tiles(case)]
        pairs = sum(n * (T - case["first"]) for n in seen)
    else:
        seen = _cross_lens(case)
        pairs = sum(n * T for n in seen)
    return {"bytes": 4 * sum(seen) * K * D + 4 * B * T * H * D + B * T * case["tiles"] + 4 * B, "flops": 4 * pairs * H * D}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "norm":
        x = s["h"].to(f64) + (0 if s["delta"] is None else s["delta"].to(f64))
        y = x / torch.sqrt(torch.mean(x ** 2, dim=1) + EPS)[:, None] * s["weight"].to(f64)[None]
        out = {} if s["delta"] is None else {"h": x}
        # the 8-bit numbers stand for y, to within their steps
        return dict(out, **{"out" if case["out"] == "bf16" else "values": y})
    if case["op"] == "rope":
        T, D, page = (case[k] for k in ("tokens", "dim", "page"))
        pairs, angle, at = D // 2, [], 0
        for axis, n in enumerate(s["sections"]):
            f = 500000.0 ** (-torch.arange(at, at + n, dtype=f64, device="cuda") / pairs)
            angle.append(s["positions"][axis].to(f64)[:, None] * f)
            at += n
        turn = torch.polar(torch.ones(T, 1, pairs, dtype=f64, device="cuda"), torch.cat(angle, 1)[:, None])

        def rotated(x):
            x = x.to(f64)
            z = torch.view_as_complex(x.view(T, -1, pairs, 2) if case["interleaved"] else
                                      x.view(T, -1, 2, pairs).transpose(2, 3).contiguous()) * turn
            z = torch.view_as_real(z)
            return (z if case["interleaved"] else z.transpose(2, 3)).reshape(x.shape)

        out = {"q": rotated(s["q"]), "k_pool": s["k_pool"].to(f64), "v_pool": s["v_pool"].to(f64)}
        rot, n = rotated(s["k"]), s["written"]
        at = s["slots"][:n].long()
        for name, x in (("k_pool", rot), ("v_pool", s["v"].to(f64))):
            flat = out[name].transpose(1, 2).reshape(-1, case["kv_heads"], D)  # [slot][head][D]
            flat[at] = x[:n]
            out[name] = flat.view(-1, page, case["kv_heads"], D).transpose(1, 2)
        return out
    H, K, D = (case[k] for k in ("heads", "kv_heads", "dim"))
    out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
    for b in range(case["batch"]):
        for h in range(K):
            if case["op"] == "paged":
                n = _lengths(case)[b]
                pages = s["page_table"][b, :-(-n // case["page"])].long()
                k, v = (s[x][pages, h].reshape(-1, D)[:n].to(f64) for x in ("k_pool", "v_pool"))
                p = torch.softmax(s["q"][b, h * (H // K):(h + 1) * (H // K)].to(f64) @ k.T / D ** 0.5, dim=1)
                out[b, h * (H // K):(h + 1) * (H // K)] = p @ v
                continue
            n = _cross_tiles(case)[b] * (case["states"] // case["tiles"]) if case["tiles"] else _cross_lens(case)[b]
            t0 = case["first"] if case["tiles"] else 0
            k, v = (s[x][b, :n, h].to(f64) for x in ("k", "v"))
            for i in range(h * (H // K), (h + 1) * (H // K)):
                out[b, t0:, i] = torch.softmax(s["q"][b, t0:, i].to(f64) @ k.T / D ** 0.5, dim=1) @ v
    return out
