"""The operators of a decode step with drafted tokens against their formulas in 64 bits.

Where the bounds come from.  A bf16 result is one rounding to nearest: 2^-8 of its value (HALF).  Heads: the sum of 128 squares runs
through 8 + 4 fp32 additions, so 1/rms is within 12/2 * 2^-24 with its root, and x * r * w adds two roundings: 2^-20 of the value;
the rotation, two products and a sum, 2^-22 of |a| + |b|; table values taken as given.  Attention: p is rounded to bf16 (2^-8 of itself)
before the product with v, and its exponent carries the fp32 error of a dot product of up to 128 terms (128 * 2^-24 * sum |q k| scale,
below 2^-11 for the sums of up to 60 here) and of exp2 (2^-22): out is within (2^-8 + 2^-10) * sum p |v| / sum p of the formula, before
its own rounding.  Sampling: every weight is within 2^-26 of itself (half a unit of 2^-26 for the polynomial's value, 2^-29 each for its fp32 roundings, the product and the
table's entry; or within a few 2^-45 of the largest), so a border of the distribution function, a quotient of two sums, lies within 2^-25 of where 64 bits
put it: a token may differ only where u or a filter's bound lies that near to one."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
HALF = 2.0 ** -8  # half the spacing of bf16's 8 significant bits, relative
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def tq():
    from paper_2509_22951_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ws(tq):
    w = tq.tq_attn_workspace()
    yield w
    assert tq.tq_attn_status(w) == 0
    torch.cuda.synchronize()
    assert int(w.buf[:2048].view(torch.int32).abs().sum()) == 0  # every call left the counters as it found them


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def f32(x):
    return torch.tensor(x, dtype=F32, device="cuda")


def within(got, ref, bound):
    err = (got.to(F64) - ref).abs()
    assert bool((err <= bound).all()), (float((err - bound).max()), float(err.max()))


# ------------------------------------------------------------------------------------------------ heads
def rope_table(n, rot):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=F64, device="cuda") / rot)
    a = torch.arange(n, dtype=F64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def heads_ref(x, w, eps, table, positions, sections, interleaved):
    """x [T][n][D]; -> (normalised and rotated, sum of the magnitudes that went into each element)"""
    x = x.to(F64)
    x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.to(F64)
    R = table.shape[1]
    axis = torch.tensor([a for a, n in enumerate(sections) for _ in range(n)], device="cuda")
    row = positions[axis].long().t()
    i = torch.arange(R // 2, device="cuda")
    c, s = table.to(F64)[row, i][:, None], table.to(F64)[row, R // 2 + i][:, None]
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, R // 2 + i)
    out, mag = x.clone(), x.abs()
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
    mag[..., ia] = mag[..., ib] = a.abs() + b.abs()
    return out, mag


@pytest.mark.parametrize("H,K,D,rot", [(4, 2, 128, 128), (3, 1, 64, 64), (6, 6, 128, 64), (5, 1, 64, 8), (24, 8, 128, 120)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("xt", [F32, BF])
@pytest.mark.parametrize("T,axes", [(1, 1), (5, 3), (333, 2), (400, 3)])
def test_qk_norm_rope_append(tq, H, K, D, rot, interleaved, xt, T, axes):
    g = gen(T + H + rot)
    page = 24
    sections = {1: [rot // 2], 2: [rot // 2 - 3, 3], 3: [1, rot // 2 - 1, 0]}[axes]
    pages = T // page + 3
    kp, vp = (randn(g, pages, page, K, D, dtype=BF).transpose(1, 2) if T % 2 else randn(g, pages, K, page, D, dtype=BF) for _ in range(2))
    cache = tq.tq_kv_cache(kp, vp)
    wide = randn(g, T, (H + 2 * K) * D + 8, dtype=xt, scale=5)  # q, k, v side by side, as one product leaves them
    q, k, v = wide[:, :H * D], wide[:, H * D:(H + K) * D], wide[:, (H + K) * D:(H + 2 * K) * D]
    qw, kw = randn(g, D, scale=0.3) + 1, randn(g, D, scale=0.3) + 1
    table = rope_table(500, rot)
    pos = torch.randint(0, 500, (axes, T), generator=g, device="cuda", dtype=torch.int32)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T].int()
    slots[T // 2] = -1
    want_k, want_v = kp.to(F64).clone(), vp.to(F64).clone()
    keep = slots >= 0
    at = slots[keep].long()
    rk, mk = heads_ref(k.reshape(T, K, D), kw, 1e-5, table, pos, sections, interleaved)
    bound_k = torch.zeros_like(want_k)
    want_k[at // page, :, at % page] = rk[keep]
    bound_k[at // page, :, at % page] = rk[keep].abs() * HALF + mk[keep] * 2.0 ** -19
    want_v[at // page, :, at % page] = v.reshape(T, K, D)[keep].to(BF).to(F64)
    out = tq.tq_qk_norm_rope_append(q, k, v, qw, kw, table, pos, slots, cache, eps=1e-5, sections=sections, interleaved=interleaved)
    rq, mq = heads_ref(q.reshape(T, H, D), qw, 1e-5, table, pos, sections, interleaved)
    within(out, rq, rq.abs() * HALF + mq * 2.0 ** -19)
    within(kp, want_k, bound_k)
    assert torch.equal(vp.to(F64), want_v)
    assert tq.tq_kv_cache_status(cache) == 0


def test_heads_of_zeros_and_what_is_not_finite(tq):
    g = gen(4)
    kp, vp = randn(g, 2, 2, 16, 64, dtype=BF), randn(g, 2, 2, 16, 64, dtype=BF)
    cache = tq.tq_kv_cache(kp, vp)
    q, k, v = randn(g, 3, 4, 64), randn(g, 3, 2, 64), randn(g, 3, 2, 64)
    q[0, 1] = 0
    k[1, 0, 7] = NAN
    q[2, 3, 60] = INF
    w = torch.ones(64, device="cuda")
    out = tq.tq_qk_norm_rope_append(q, k, v, w, w, rope_table(10, 32), i32([1, 2, 3]), i32([0, 1, 17]), cache)
    assert not out[0, 1].any() and bool(out[2, 3, 60].isnan()) and not out[2, 3, 32:60].any() and bool(out[2, :3].isfinite().all())
    assert bool(kp[0, 0, 1].isnan().all()) and bool(kp[0, 1, 1].isfinite().all()) and torch.equal(vp[1, :, 1], v[2].to(BF))
    # positions and slots out of range, as without the norm
    k0, v0 = kp.clone(), vp.clone()
    out = tq.tq_qk_norm_rope_append(q[:1], k[:1], v[:1], w, w, rope_table(10, 64), i32([10]), i32([3]), cache)
    assert bool(out.isnan().all()) and tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_POSITION
    out = tq.tq_qk_norm_rope_append(q[:1], k[:1], v[:1], w, w, rope_table(10, 64), i32([9]), i32([32]), cache)
    assert bool(out.isfinite().all()) and tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_PAGE
    assert torch.equal(kp.view(torch.int16), k0.view(torch.int16)) and torch.equal(vp, v0)
    assert tq.tq_qk_norm_rope_append(q[:0], k[:0], v[:0], w, w, rope_table(10, 64), i32([]), i32([]), cache).shape == (0, 4, 64)


# ------------------------------------------------------------------------------------------------ attention
def attend_ref(q, k, v, seen, scale):
    """q [n][D], k / v [m][D], seen [n][m] -> out, lse, bound of out; what is not seen is not touched."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    x = torch.where(seen, q @ torch.where(seen.any(0)[:, None], k, 0.0).t() * scale, -INF)
    lse = torch.logsumexp(x, -1) if x.shape[1] else torch.full((q.shape[0],), -INF, dtype=F64, device=q.device)
    p = torch.where(seen, torch.exp(x - torch.where(lse.isfinite(), lse, 0.0)[:, None]), 0.0)
    vs = torch.where(seen.any(0)[:, None], v, 0.0)
    out = p @ vs
    return out, lse, (p @ vs.abs()) * (HALF + 2.0 ** -10) + out.abs() * HALF + 1e-30


def check_lse(got, want):
    empty = want == -INF
    assert torch.equal(got == -INF, empty)
    within(got[~empty], want[~empty], 2.0 ** -11 + want[~empty].abs() * 2.0 ** -20)


def pack(bits, words):
    """Rows of booleans -> int32 words."""
    n = bits.shape[1]
    w = torch.zeros(bits.shape[0], words * 32, dtype=torch.int64)
    w[:, :n] = bits.long()
    w = (w.view(-1, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).int().cuda()


def tree_bits(n, rng):
    """Ancestors and self, each token after an earlier one."""
    bits = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        if i:
            bits[i] = bits[rng.randrange(max(0, i - 5), i)]
        bits[i, i] = True
    return bits


def tree_case(tq, ws, new, lens, H, K, D, page, kind, seed, layout=0, lead=0, tail=0, spoil=True, words=None, q_pad=0):
    """new[b] new tokens, lens[b] states with them; kind: chain, tree, random (rows that see none of the new tokens among them)."""
    g, rng = gen(seed), random.Random(seed)
    B = len(lens)
    need = [-(-max(n, 0) // page) for n in lens]
    pool = sum(need) + 2
    shape = (pool, K, page, D) if layout == 0 else (pool, page, K, D)
    kp, vp = randn(g, *shape, dtype=BF), randn(g, *shape, dtype=BF)
    if layout:
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    perm = torch.randperm(pool, generator=g, device="cuda")
    table = torch.full((B, max(max(need), 1)), -7, dtype=torch.int32, device="cuda")  # entries past a length are not followed
    used = torch.zeros(pool, page, dtype=torch.bool, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n].int()
        if lens[b] > 0:
            used[perm[at:at + n]] = (torch.arange(n * page, device="cuda") < lens[b]).view(n, page)
        at += n
    if spoil:  # slots that no length reaches hold NaN and infinities
        kp.masked_fill_(~used[:, None, :, None], NAN)
        vp.masked_fill_(~used[:, None, :, None], INF)
    first = [lead]
    for n in new:
        first.append(first[-1] + n)
    T = first[-1] + tail
    bits, mask = [], None
    for n in new:
        bits.append(torch.ones(n, n).tril().bool() if kind == "chain" else tree_bits(n, rng) if kind == "tree" else torch.rand(n, n) < 0.3)
        if kind == "random" and n > 1:
            bits[-1][n // 2] = False
    if kind != "chain":
        words = -(-max(new + [1]) // 32) if words is None else words
        mask = torch.full((T, words), -1, dtype=torch.int32, device="cuda")  # bits past a sequence's tokens mean nothing
        for b, n in enumerate(new):
            ones = torch.ones(n, 32 * words, dtype=torch.bool)
            ones[:, :n] = bits[b][:, :32 * words]
            mask[first[b]:first[b + 1]] = pack(ones, words)
            bits[b][:, 32 * words:] = False
    q = randn(g, T, H * D + q_pad, dtype=BF, scale=1.5)[:, :H * D].view(T, H, D) if q_pad == 0 else \
        randn(g, T, H * D + q_pad, dtype=BF, scale=1.5)[:, :H * D].unflatten(1, (H, D))
    cache = tq.tq_kv_cache(kp, vp)
    ft, lt = i32(first), i32(lens)
    out, lse = torch.full((T, H, D), 7.0, dtype=BF, device="cuda"), torch.full((T, H), 7.0, device="cuda")
    tq.tq_tree_attention(q, cache, table, ft, lt, ws, mask=mask, out=out, lse=lse)
    again = tq.tq_tree_attention(q, cache, table, ft, lt, ws, mask=mask, out=torch.full_like(out, 7.0))
    assert torch.equal(out, again)  # the same call, the same bits
    assert bool((out[:lead] == 7).all()) and bool((out[first[-1]:] == 7).all()) and bool((lse[first[-1]:] == 7).all())  # rows of no sequence
    at = 0
    for b, n in enumerate(need):
        ids = perm[at:at + n]
        at += n
        length, rows = max(lens[b], 0), slice(first[b], first[b + 1])
        m = new[b]
        seen = torch.ones(m, length, dtype=torch.bool, device="cuda")
        own = min(m, length)
        if own:
            seen[:, length - own:] = bits[b][:, m - own:].cuda()
        for h in range(K):
            k, v = (x[ids, h].reshape(-1, D)[:length] for x in (kp, vp))
            for i in range(h * (H // K), (h + 1) * (H // K)):
                want, wl, bound = attend_ref(q[rows, i], k, v, seen, D ** -0.5)
                within(out[rows, i], want, bound)
                check_lse(lse[rows, i], wl)
    assert tq.tq_kv_cache_status(cache) == 0
    return cache


@pytest.mark.parametrize("kind", ["chain", "tree", "random"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,K", [(4, 4), (6, 2), (8, 1), (24, 8), (20, 2)])
@pytest.mark.parametrize("new,lens,page", [([1], [1], 16), ([5], [37], 16), ([7, 0, 3, 1], [64, 0, 65, 1], 1), ([16, 15, 2, 33, 9], [500, 15, 16, 127, 129], 24),
                                           ([31, 8, 1], [2500, 128, 257], 64), ([4, 70], [130, 200], 200)])
def test_tree_attention(tq, ws, kind, D, H, K, new, lens, page):
    tree_case(tq, ws, new, lens, H, K, D, page, kind, seed=sum(lens) + H, layout=(H + page) % 2)


def test_rows_of_no_sequence_are_left_alone(tq, ws):
    tree_case(tq, ws, [3, 9], [40, 300], 8, 2, 64, 16, "tree", seed=5, lead=2, tail=5)
    tree_case(tq, ws, [3, 9], [40, 300], 8, 2, 128, 16, "chain", seed=6, lead=130, tail=200)
    tree_case(tq, ws, [0, 0], [40, 0], 8, 2, 64, 16, "chain", seed=7, tail=3)


@pytest.mark.parametrize("H,K,D", [(8, 2, 64), (32, 8, 128), (12, 1, 64)])
def test_pieces_of_prompts(tq, ws, H, K, D):
    tree_case(tq, ws, [300, 1, 129], [1000, 600, 129], H, K, D, 32, "chain", seed=8, q_pad=24)


def test_wide_trees(tq, ws):
    tree_case(tq, ws, [200, 64, 65], [900, 64, 400], 8, 2, 64, 16, "tree", seed=9)
    tree_case(tq, ws, [100, 40], [900, 64], 8, 2, 128, 16, "random", seed=10, words=2)  # tokens past the words are not seen


@pytest.mark.parametrize("kind", ["chain", "tree", "random"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,K", [(8, 2), (6, 1), (5, 5)])
@pytest.mark.parametrize("new,lens,page", [([65], [65], 16), ([129], [5000], 24), ([300, 0, 131, 170], [700, 9, 131, 2900], 64), ([140, 1, 150], [140, 5000, 12000], 1), ([150, 140, 133], [64, 0, -3], 16)])
def test_tiles_of_256_rows(tq, ws, kind, D, H, K, new, lens, page):
    tree_case(tq, ws, new, lens, H, K, D, page, kind, seed=sum(lens) + H, layout=page % 2)


def test_fewer_states_than_new_tokens(tq, ws):
    tree_case(tq, ws, [9, 5, 4], [4, 0, -3], 4, 2, 64, 16, "chain", seed=11)
    tree_case(tq, ws, [9, 5, 40], [4, 0, 33], 4, 2, 64, 16, "random", seed=12)


def test_tree_attention_many_sequences(tq, ws):
    rng = random.Random(3)
    new = [rng.choice([0, 1, 1, 2, 5, 8]) for _ in range(600)]
    tree_case(tq, ws, new, [n + rng.randrange(0, 300) for n in new], 4, 2, 64, 16, "tree", seed=13)


def test_tree_attention_long(tq, ws):
    tree_case(tq, ws, [12, 3], [100003, 5], 8, 2, 128, 48, "tree", seed=14)
    tree_case(tq, ws, [40], [50001], 32, 2, 64, 64, "chain", seed=15)


def test_one_new_token_is_paged_attention(tq, ws):
    g = gen(16)
    lens, H, K, D, page = [1, 700, 129, 64], 8, 2, 64, 16
    kp, vp = randn(g, 80, K, page, D, dtype=BF), randn(g, 80, K, page, D, dtype=BF)
    cache, q = tq.tq_kv_cache(kp, vp), randn(g, 4, H, D, dtype=BF)
    table = torch.randint(0, 80, (4, 44), generator=g, device="cuda", dtype=torch.int32)
    a = tq.tq_paged_attention(q, cache, table, i32(lens), ws).to(F64)
    b = tq.tq_tree_attention(q, cache, table, i32([0, 1, 2, 3, 4]), i32(lens), ws).to(F64)
    within(b, a, a.abs().amax(-1, keepdim=True) * 2 * (2 * HALF + 2.0 ** -10))


def test_large_scores(tq, ws):
    """Scores of several hundred: one state takes all the weight, whatever came before it in the running maximum."""
    g = gen(17)
    kp, vp = randn(g, 40, 1, 32, 64, dtype=BF), randn(g, 40, 1, 32, 64, dtype=BF)
    q = randn(g, 3, 2, 64, dtype=BF)
    kp[3, 0, 7] = q[0, 0] * 60
    kp[36, 0, 1] = q[0, 0] * 70
    kp[5, 0, 9] = q[0, 1] * -80
    kp[20, 0, 9] = q[2, 1] * 50
    table = torch.arange(40, device="cuda", dtype=torch.int32)[None].contiguous()
    out = tq.tq_tree_attention(q, tq.tq_kv_cache(kp, vp), table, i32([0, 3]), i32([1280]), ws)
    k, v = kp.flatten(0, 2).to(F64), vp.flatten(0, 2).to(F64)
    for i in range(3):
        x = q[i].to(F64) @ k[:1278 + i].t() / 8
        w = torch.softmax(x, 1)
        # the exponent's error grows with the score: 2^-24 * 64 * sum |q k| / 8, below 2^-7 here
        within(out[i], w @ v[:1278 + i], (w @ v[:1278 + i].abs()) * (HALF + 2.0 ** -6) + 2.0 ** -8)


def test_states_that_a_token_does_not_see_may_hold_anything(tq, ws):
    g = gen(18)
    for D, H, K, n, length in ((64, 4, 2, 6, 131), (128, 16, 2, 20, 700), (128, 8, 1, 30, 700), (64, 16, 2, 31, 900)):
        kp, vp = randn(g, 60, K, 16, D, dtype=BF), randn(g, 60, K, 16, D, dtype=BF)
        q = randn(g, n, H, D, dtype=BF)
        table = torch.randperm(60, generator=g, device="cuda").int()[None].contiguous()
        slot = lambda s: (int(table[0, s // 16]), slice(None), s % 16)  # noqa: E731
        bits = torch.ones(n, n).tril().bool()
        bits[:, 2] = bits[:, 3] = False  # new tokens 2 and 3 see themselves alone, nobody else sees them
        bits[2, 2] = bits[3, 3] = True
        cache = tq.tq_kv_cache(kp, vp)
        args = (q, cache, table, i32([0, n]), i32([length]), ws)
        clean = tq.tq_tree_attention(*args, mask=pack(bits, 1))
        kp[slot(length - n + 2)] = NAN
        vp[slot(length - n + 2)] = INF
        vp[slot(length - n + 3)] = -INF
        lse = torch.empty(n, H, device="cuda")
        out = tq.tq_tree_attention(*args, mask=pack(bits, 1), lse=lse)
        others = [i for i in range(n) if i not in (2, 3)]
        within(out[others], clean[others].to(F64), clean[others].to(F64).abs().amax(-1, keepdim=True) * 2 * (2 * HALF + 2.0 ** -10))
        assert bool(lse[others].isfinite().all())
        assert bool(out[2].isnan().all()) and bool((out[3] == -INF).all())
        # in a chain the tokens before them do not see them either
        out = tq.tq_tree_attention(*args)
        ref = tq.tq_tree_attention(q[:2], cache, table, i32([0, 2]), i32([length - n + 2]), ws)
        within(out[:2], ref.to(F64), ref.to(F64).abs().amax(-1, keepdim=True) * 2 * (2 * HALF + 2.0 ** -10))
        assert bool(out[2:].isnan().all())


def test_a_broken_query_stays_by_itself(tq, ws):
    g = gen(19)
    kp, vp = randn(g, 30, 2, 16, 64, dtype=BF), randn(g, 30, 2, 16, 64, dtype=BF)
    q = randn(g, 8, 4, 64, dtype=BF)
    table = torch.arange(30, device="cuda", dtype=torch.int32)[None].contiguous()
    args = (tq.tq_kv_cache(kp, vp), table, i32([0, 8]), i32([470]), ws)
    clean = tq.tq_tree_attention(q, *args)
    q[3, 1, 5] = NAN
    out = tq.tq_tree_attention(q, *args)
    assert bool(out[3, 1].isnan().all())
    keep = torch.ones(8, 4, dtype=torch.bool, device="cuda")
    keep[3, 1] = False
    assert torch.equal(out[keep], clean[keep])


def test_pages_lengths_and_rows_out_of_range(tq, ws):
    g = gen(20)
    kp, vp = randn(g, 6, 1, 16, 64, dtype=BF), randn(g, 6, 1, 16, 64, dtype=BF)
    cache, q = tq.tq_kv_cache(kp, vp), randn(g, 6, 2, 64, dtype=BF)
    k, v = kp[:, 0], vp[:, 0]
    # a page outside the pool hides its states, a length past the table is cut there
    out = tq.tq_tree_attention(q, cache, i32([[0, 6, 2], [1, 3, -1]]), i32([0, 3, 6]), i32([48, 60]), ws)
    assert tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_PAGE
    for rows, pages, seen in ((slice(0, 3), [0, 2], [[True] * (30 + i) + [False] * (2 - i) for i in range(3)]), (slice(3, 6), [1, 3], [[True] * 32] * 3)):
        seen = torch.tensor(seen, device="cuda")
        for h in range(2):
            want, _, bound = attend_ref(q[rows, h], k[pages].reshape(-1, 64), v[pages].reshape(-1, 64), seen, 0.125)
            within(out[rows, h], want, bound)
    assert tq.tq_kv_cache_status(cache) == 0
    # rows outside the batch are clamped to it
    out = torch.full((6, 2, 64), 7.0, dtype=BF, device="cuda")
    tq.tq_tree_attention(q, cache, i32([[0, 1, 2]] * 3), i32([-5, 2, 2 ** 31 - 1, 3]), i32([30, 40, 20]), ws, out=out)
    assert bool(out.isfinite().all()) and not bool((out == 7).all(-1).any())
    assert tq.tq_tree_attention(q[:0], cache, i32([[0]]), i32([0, 0]), i32([4]), ws).shape == (0, 2, 64)


def test_offsets_past_32_bits(tq, ws):
    g = gen(21)
    K, page, D, H, far = 2, 16, 64, 4, 2 ** 32 // (2 * 16 * 64) + 11
    pool = torch.empty((far + 1) * K * page * D, dtype=BF, device="cuda")
    kp = pool.view(far + 1, K, page, D)
    pages = [far, 3, far - 2, 0]
    kp[pages] = randn(g, 4, K, page, D, dtype=BF)
    cache = tq.tq_kv_cache(kp, kp)
    q = randn(g, 5, H, D, dtype=BF)
    table = i32([pages])
    out = tq.tq_tree_attention(q, cache, table, i32([0, 5]), i32([64]), ws)
    seen = torch.ones(5, 64, device="cuda").tril(59).bool()
    for h in range(H):
        k = kp[pages, h // 2].reshape(-1, D)
        want, _, bound = attend_ref(q[:, h], k, k, seen, 0.125)
        within(out[:, h], want, bound)
    # the last token's keys and values move down two places, from one page that far to another
    before = kp[pages].clone()
    tokens, path, count, lens = tq.tq_tree_accept(tq.tq_kv_caches([cache]), i32([[3, far, far - 2, 0]]), i32([0, 4]), i32([33]), i32([9, 9, 9, 8]), i32([-1, 0, 0, 0]),
                                                  i32([8, 0, 0, 5]), 4)
    assert tokens.tolist() == [[8, 5, -1, -1]] and path.tolist() == [[0, 3, -1, -1]] and count.tolist() == [2] and lens.tolist() == [31]
    before[0, :, 14] = before[2, :, 0]
    assert torch.equal(kp[pages], before)


def test_streams_and_graphs(tq):
    g = gen(22)
    kp, vp = randn(g, 200, 2, 16, 128, dtype=BF), randn(g, 200, 2, 16, 128, dtype=BF)
    cache = tq.tq_kv_cache(kp, vp)
    table = torch.randperm(200, generator=g, device="cuda").int().view(2, 100)
    first, lens, u = i32([0, 12, 20]), i32([1600, 777]), torch.rand(20, generator=g, device="cuda")
    q, x = randn(g, 20, 8, 128, dtype=BF), randn(g, 20, 5000, scale=3)
    parents, drafted = i32([-1] + list(range(11)) + [-1] + list(range(7))), torch.randint(0, 40, (20,), generator=g, device="cuda").int()

    def step(w, stream=None):
        o = tq.tq_tree_attention(q, cache, table, first, lens, w, stream=stream)
        t, lp = tq.tq_sample(x, u, top_k=torch.full_like(drafted, 40), logprob=True, stream=stream) if stream is None else tq.tq_sample(x, u, logprob=True, stream=stream)
        return o, t, lp, *tq.tq_tree_accept(None, None, first, lens, drafted, parents, t % 40, 6, stream=stream)

    w = [tq.tq_attn_workspace() for _ in range(3)]
    want, plain = step(w[0]), None
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for rep in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got.append(step(w[1 + i]))
    torch.cuda.synchronize()
    for o in got:
        assert all(torch.equal(a, b) for a, b in zip(o, want))
    other = tq.tq_tree_attention(q, cache, table, first, lens, w[1], stream=streams[0])
    torch.cuda.synchronize()
    assert torch.equal(other, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(w[0])
    q2, x2 = randn(g, 20, 8, 128, dtype=BF), randn(g, 20, 5000, scale=3)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    q.copy_(q2), x.copy_(x2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, step(w[1])))


# ------------------------------------------------------------------------------------------------ sampling
def sample_ref(x, u, t=None, k=None, p=None, m=None):
    """-> tokens, logprobs, and how near (as a share of the kept sum) u or a bound lies to a border: nearer than 2^-25 either side may be taken."""
    out, lps, near = [], [], []
    for r in range(x.shape[0]):
        v = x[r].to(F64)
        v = torch.where(v.isnan(), -INF, v)
        T = 1.0 if t is None else float(t[r])
        value, place = v.sort(descending=True, stable=True)
        if float(value[0]) == -INF:
            out.append(-1), lps.append(-INF), near.append(1.0)
            continue
        if not T > 0:
            out.append(int(place[0])), lps.append(0.0), near.append(1.0)
            continue
        w = torch.exp((value - value[0]) / T) if float(value[0]) < INF else torch.zeros_like(value)
        w[value == value[0]] = 1.0
        n, gap = w.numel(), 1.0
        if k is not None and 0 < int(k[r]) < n:
            n = int(k[r])
        w = w[:n]
        if p is not None and float(p[r]) < 1:
            before = w.cumsum(0) - w
            off = (before - float(p[r]) * w.sum()) / w.sum()
            n = max(1, int((off < 0).sum()))
            gap = float(off[1:].abs().min()) if off.numel() > 1 else 1.0
        if m is not None and float(m[r]) > 0:
            n = max(1, min(n, int((w >= float(m[r])).sum())))
        ids, order = place[:n].sort()
        c = w[:n][order].cumsum(0)
        target = max(0.0, float(u[r])) * c[-1]
        at = min(int((c <= target).sum()), int((c < c[-1]).sum()))
        gap = min(gap, float((c / c[-1] - target / c[-1]).abs().min()))
        out.append(int(ids[at])), lps.append(float((w[:n][order][at] / c[-1]).log())), near.append(gap)
    return torch.tensor(out), torch.tensor(lps, dtype=F64), torch.tensor(near, dtype=F64)


def sample_case(tq, x, u, **kw):
    token, logprob = tq.tq_sample(x, u, logprob=True, **kw)
    assert torch.equal(token, tq.tq_sample(x, u, **kw))
    names = {"temperature": "t", "top_k": "k", "top_p": "p", "min_p": "m"}
    want, lp, near = sample_ref(x, u, **{names[n]: v for n, v in kw.items()})
    token, logprob = token.cpu(), logprob.cpu().to(F64)
    same = token == want
    assert bool((same | (near < 2.0 ** -25)).all()), (token[~same], want[~same], near[~same])
    lp, got = lp[same], logprob[same]
    none = lp == -INF
    assert torch.equal(got == -INF, none)
    err = (got - lp)[~none].abs()
    # two roundings of the result, and the sum's own 2^-26 with the logarithm's 2^-29
    assert bool((err <= lp[~none].abs() * 2.0 ** -23 + 2.0 ** -25).all()), float(err.max())
    return token


def logits(g, rows, vocab, floor=1.5, top=15.0, dtype=F32):
    x = randn(g, rows, vocab, scale=floor)
    n = min(vocab, 100)
    at = torch.randint(0, vocab, (rows, n), generator=g, device="cuda")
    x.scatter_add_(1, at, top * torch.rand(rows, 1, generator=g, device="cuda") - 1.5 * torch.arange(1, n + 1, device="cuda").log()[None])
    return x.to(dtype)


VOCABS = [1, 2, 3, 31, 1000, 1024, 4095, 4097, 16383, 16384, 50257, 128256, 262144]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("vocab", VOCABS)
def test_sample(tq, vocab, dtype):
    g, R = gen(vocab), 24 if vocab < 100000 else 10
    x, u = logits(g, R, vocab, dtype=dtype), torch.rand(R, generator=g, device="cuda")
    rng = random.Random(vocab)
    each = lambda *c: [rng.choice(c) for _ in range(R)]  # noqa: E731
    sample_case(tq, x, u)
    sample_case(tq, x, u, temperature=f32(each(0.1, 0.7, 1.0, 3.0, 50.0)))
    sample_case(tq, x, u, top_k=i32(each(1, 2, 7, 50, 300, 1100, 3000, vocab, vocab - 1, 0, -1)))
    sample_case(tq, x, u, top_p=f32(each(0.01, 0.3, 0.9, 0.999, 1.0, 1.5)))
    sample_case(tq, x, u, min_p=f32(each(0.0, 0.001, 0.1, 0.9, 1.0)))
    sample_case(tq, x, u, temperature=f32(each(0.0, -1.0, 0.3, 1.0, 2.0)), top_k=i32(each(0, 1, 5, 40, 1000, 5000)), top_p=f32(each(0.2, 0.8, 0.95, 1.0)),
                min_p=f32(each(0.0, 0.0, 0.01, 0.2)))


def test_sample_of_equals(tq):
    """Ties at every border: the lowest index is taken first."""
    g, R, V = gen(30), 16, 3001
    u = torch.rand(R, generator=g, device="cuda")
    for x in (torch.zeros(R, V, device="cuda"), torch.randint(-3, 3, (R, V), generator=g, device="cuda").float(), torch.randint(0, 2, (R, V), generator=g, device="cuda").float() * -0.0,
              torch.full((R, 70000), -2.5, device="cuda", dtype=BF)):
        sample_case(tq, x, u)
        sample_case(tq, x, u, top_k=i32([1, 2, 3, 10, 100, 500, 501, 1023, 1024, 1025, 1500, 2047, 2048, 2049, 2999, 3000]))
        sample_case(tq, x, u, top_p=f32([0.1 + 0.05 * r for r in range(R)]))
        sample_case(tq, x, u, min_p=f32([0.0, 0.1, 0.5, 0.9999, 1.0, 1.0000001, 2.0, INF] * 2), temperature=f32([0.7] * R))
        sample_case(tq, x, u, top_k=i32([700] * R), top_p=f32([0.1 + 0.05 * r for r in range(R)]), temperature=f32([0.5] * R))
        assert sample_case(tq, x, u, temperature=f32([0.0] * R)).tolist() == [int((r == r.max()).nonzero()[0]) for r in x]


@pytest.mark.parametrize("vocab,scale", [(2500, 0.02), (30000, 1.0), (128256, 0.3), (128256, 1.5), (262144, 1.0), (262144, 2.5)])
def test_sample_where_the_border_is_crowded(tq, vocab, scale):
    """Top-p among few, hundreds and thousands of weights next to one another, distinct and (16 bits) in groups of equals, with and without min-p."""
    g, R = gen(vocab + 1), 12
    u, p = torch.rand(R, generator=g, device="cuda"), f32([0.02, 0.1, 0.3, 0.5, 0.7, 0.8, 0.9, 0.95, 0.97, 0.99, 0.999, 0.9999])
    for dtype in (F32, BF):
        x = randn(g, R, vocab, dtype=dtype, scale=scale)
        for t in (0.4, 1.0):
            sample_case(tq, x, u, temperature=f32([t] * R), top_p=p)
        sample_case(tq, x, u, top_p=p, min_p=f32([0.0, 1e-3, 0.2] * (R // 3)))
        # the draw at the far end is the last kept token: a border one place off shows
        sample_case(tq, x, torch.full((R,), 1.0 - 2.0 ** -24, device="cuda"), top_p=p)
    x[:, ::7] = x[:, :1]  # a seventh of the row is one logit
    sample_case(tq, x, u, top_p=p)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("scale", [0.5, 3.0])
def test_sample_of_the_first_hundreds(tq, dtype, scale):
    """Lists of more than 128 tokens: distinct logits, and (16 bits) groups of equals that no part of the list holds."""
    g, R = gen(int(scale * 10)), 12
    x, u = randn(g, R, 60000, dtype=dtype, scale=scale), torch.rand(R, generator=g, device="cuda")
    k, last = i32([129, 200, 300, 500, 700, 900, 1000, 1023, 1024, 150, 400, 600]), torch.full((R,), 1.0 - 2.0 ** -24, device="cuda")
    p, t = f32([0.1, 0.3, 0.5, 0.7, 0.9, 0.95, 0.99, 0.999, 1.0, 0.9, 0.9, 0.9]), f32([0.3, 1.0, 2.0] * 4)
    for v in (u, last, u * 0):
        sample_case(tq, x, v, top_k=k, temperature=t)
        sample_case(tq, x, v, top_k=k, top_p=p)
        sample_case(tq, x, v, top_k=k, top_p=p, min_p=f32([0.0, 0.01, 0.3] * 4), temperature=t)
    x[:, ::60] = x.amax() + 1  # a thousand equals at the head
    sample_case(tq, x, u, top_k=k, top_p=p)


def test_sample_of_what_is_not_finite(tq):
    g, V = gen(31), 20000
    x = logits(g, 12, V)
    x[0] = -INF
    x[1] = NAN
    x[2, ::2] = NAN
    x[3, 5:] = -INF
    x[4, 77] = INF
    x[5, [9, 19999, 4]] = INF
    x[6, :-1] = -INF
    x[7, 100] = 3e38
    x[8] = -3e38
    x[9] *= 1e30
    x[10] = 1e-40 * torch.arange(V, device="cuda")
    u = torch.rand(12, generator=g, device="cuda")
    got = sample_case(tq, x, u)
    assert got[0] == -1 and got[1] == -1 and got[4] == 77 and got[6] == V - 1 and got[7] == 100 and int(got[2]) % 2 == 1
    got = sample_case(tq, x, u, temperature=f32([0.0] * 12))
    assert got[0] == -1 and got[1] == -1 and got[4] == 77 and got[5] == 4
    for kw in (dict(top_k=i32([2] * 12)), dict(top_p=f32([0.7] * 12)), dict(min_p=f32([0.3] * 12)), dict(top_k=i32([30] * 12), top_p=f32([0.5] * 12), min_p=f32([0.01] * 12))):
        sample_case(tq, x, u, **kw)
    # settings at their ends: NaN is as good as none, and temperatures of any size
    y = logits(g, 8, V)
    u = torch.rand(8, generator=g, device="cuda")
    t = f32([1e-30, 1e-3, 1e-45, 1e30, 3e38, INF, NAN, -0.0])
    sample_case(tq, y, u, temperature=t)
    sample_case(tq, y, u, temperature=t, top_k=i32([5] * 8), top_p=f32([0.9] * 8))
    nan = f32([NAN] * 8)
    assert torch.equal(tq.tq_sample(y, u, top_p=nan, min_p=nan), tq.tq_sample(y, u))
    sample_case(tq, y, u, top_p=f32([0.0, -1.0, 1e-30, 2.0, INF, -INF, 0.5, 1.0]))
    sample_case(tq, y, u, min_p=f32([0.0, -1.0, 1e-30, 2.0, INF, -INF, 0.5, 1.0]))


def test_sample_at_the_ends_of_u(tq):
    g, V = gen(32), 9000
    x = logits(g, 6, V)
    x[:, :3] = -INF
    x[:, -3:] = -INF
    u = f32([0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, NAN])
    assert tq.tq_sample(x, u).tolist() == [3, V - 4, V - 4, V - 4, 3, 3]
    sample_case(tq, x[:3], u[:3], top_k=i32([10] * 3))
    assert tq.tq_sample(x[:0], u[:0]).shape == (0,)


def test_sample_strides_and_alignment(tq):
    g = gen(33)
    for dtype, pitch, at, V in ((F32, 1003, 1, 1000), (F32, 40004, 3, 40000), (BF, 40003, 5, 40001), (BF, 128264, 8, 128256), (F32, 128260, 0, 128256)):
        base = randn(g, 5 * pitch + at, dtype=dtype, scale=3)
        x = base.as_strided((5, V), (pitch, 1), at)
        u = torch.rand(5, generator=g, device="cuda")
        sample_case(tq, x, u, top_k=i32([20, 0, 100, 3, 1]), top_p=f32([0.9, 0.5, 1.0, 0.99, 0.3]))
        assert torch.equal(tq.tq_sample(x, u), tq.tq_sample(x.contiguous(), u))
        one = base.as_strided((5, V), (0, 1), at)  # every row the same logits
        sample_case(tq, one, u)


def test_sample_draws_as_often_as_the_weights_say(tq):
    g, R = gen(34), 20000
    x = f32([0.0, 1.0, -1.0, 2.0, -INF, 0.5]).expand(R, 6)
    u = torch.rand(R, generator=g, device="cuda")
    n = torch.bincount(tq.tq_sample(x, u, temperature=torch.full((R,), 2.0, device="cuda")).long(), minlength=6).to(F64) / R
    want = torch.softmax(x[0].to(F64) / 2, 0)
    assert bool(((n - want).abs() <= 5 * (want * (1 - want) / R).sqrt()).all())  # five standard deviations


# ------------------------------------------------------------------------------------------------ what is accepted
def accept_ref(new, lens, tokens, parents, sampled, max_path):
    path, drawn, count, out_lens, f = [], [], [], [], 0
    for n, length in zip(new, lens):
        p = [0] if n else []
        while p and len(p) < max_path:
            after = [c for c in range(p[-1] + 1, n) if parents[f + c] == p[-1] and tokens[f + c] == sampled[f + p[-1]]]
            if not after:
                break
            p.append(after[0])
        path.append(p + [-1] * (max_path - len(p)))
        drawn.append([sampled[f + c] for c in p] + [-1] * (max_path - len(p)))
        count.append(len(p))
        out_lens.append(length - n + len(p))
        f += n
    return drawn, path, count, out_lens


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("new,lens,K,D,page,layers,max_path", [
    ([1], [1], 1, 64, 16, 1, 1), ([9, 0, 30, 5], [40, 7, 31, 5], 2, 128, 16, 3, 16), ([64] * 9, [70 + b for b in range(9)], 8, 64, 24, 2, 5),
    ([700, 33], [900, 800], 2, 64, 64, 2, 200), ([12] * 300, [20 + b % 50 for b in range(300)], 1, 64, 1, 1, 16), ([20, 20], [500, 600], 8, 128, 32, 16, 256),
])
def test_tree_accept(tq, layout, new, lens, K, D, page, layers, max_path):
    g, rng = gen(sum(lens) + layers), random.Random(sum(new) + K)
    B, need = len(new), [-(-n // page) for n in lens]
    pool = sum(need) + 1
    shape = (layers, pool, K, page, D) if layout == 0 else (layers, pool, page, K, D)
    kp, vp = randn(g, *shape, dtype=BF), randn(g, *shape, dtype=BF)
    if layout:
        kp, vp = kp.transpose(2, 3), vp.transpose(2, 3)
    perm = torch.randperm(pool).tolist()
    table, at = [[-1] * max(need) for _ in new], 0
    for b, n in enumerate(need):
        table[b][:n] = perm[at:at + n]
        at += n
    first, tokens, parents, sampled = [0], [], [], []
    for b, n in enumerate(new):
        first.append(first[-1] + n)
        # a small vocabulary: many siblings with one token, of which the first counts; some parents that are never followed
        mine = [rng.randrange(max(0, i - 6), i) if i else rng.choice([-1, 0, 3]) for i in range(n)]
        for i in range(1, n):
            if rng.random() < 0.1:
                mine[i] = rng.choice([i, i + 1, n + 5, -1, -2 ** 31, 2 ** 31 - 1])
        if b % 3 == 0:
            mine = [i - 1 for i in range(n)]
        parents += mine
        tokens += [rng.randrange(2 if b % 2 else 1) for _ in range(n)]
        sampled += [rng.randrange(2) if rng.random() < 0.3 else 0 for _ in range(n)]
    want = accept_ref(new, lens, tokens, parents, sampled, max_path)
    wk, wv = kp.clone(), vp.clone()
    for pool_t, src in ((wk, kp), (wv, vp)):
        for b, p in enumerate(want[1]):
            for d, c in enumerate(p):
                if c < 0:
                    break
                s, t = lens[b] - new[b] + c, lens[b] - new[b] + d
                pool_t[:, table[b][t // page], :, t % page] = src[:, table[b][s // page], :, s % page]
    caches = [tq.tq_kv_cache(k, v) for k, v in zip(kp, vp)]
    got = tq.tq_tree_accept(tq.tq_kv_caches(caches), i32(table), i32(first), i32(lens), i32(tokens), i32(parents), i32(sampled), max_path)
    for a, w in zip(got, want):
        assert a.tolist() == w
    assert torch.equal(kp, wk) and torch.equal(vp, wv)
    assert all(tq.tq_kv_cache_status(c) == 0 for c in caches)
    assert max(want[2]) > 1 or sum(new) == 1
    alone = tq.tq_tree_accept(None, None, i32(first), i32(lens), i32(tokens), i32(parents), i32(sampled), max_path)
    assert all(torch.equal(a, b) for a, b in zip(got, alone))


def test_tree_accept_keeps_off_what_is_out_of_range(tq):
    g = gen(41)
    kp, vp = randn(g, 3, 2, 4, 64, dtype=BF), randn(g, 3, 2, 4, 64, dtype=BF)
    k0, v0 = kp.clone(), vp.clone()
    c = tq.tq_kv_cache(kp, vp)
    caches = tq.tq_kv_caches([c])
    # rows 0 and 2 of each sequence are on the path; sequence 0's page is bad, 1's target lies before the cache, 2's state past the table
    args = (i32([0, 3, 6, 9]), i32([7, 1, 14]), i32([5] * 9), i32([-1, 9, 0] * 3), i32([5, 0, 1] * 3), 4)
    tokens, path, count, lens = tq.tq_tree_accept(caches, i32([[0, 3, 1], [0, 1, 2], [0, 1, 2]]), *args)
    assert path.tolist() == [[0, 2, -1, -1]] * 3 and count.tolist() == [2, 2, 2] and lens.tolist() == [6, 0, 13] and tokens.tolist() == [[5, 1, -1, -1]] * 3
    assert torch.equal(kp, k0) and torch.equal(vp, v0) and tq.tq_kv_cache_status(c) == tq.TQ_STATUS_BAD_PAGE
    # rows outside the batch are clamped to it
    tokens, path, count, lens = tq.tq_tree_accept(None, None, i32([-4, 2, 100, 50]), i32([7, 9, 3]), i32([1] * 6), i32([-1, 0, 0, 0, 0, 0]), i32([1] * 6), 2)
    assert count.tolist() == [2, 2, 0] and lens.tolist() == [7, 7, 3] and path.tolist() == [[0, 1], [0, 1], [-1, -1]]


# ------------------------------------------------------------------------------------------------ a run of them
def test_a_decode_step_with_drafted_tokens(tq, ws):
    """Two layers of attention, with random products between them: a tree of drafted tokens gives what the tokens one by one give, and what is
    accepted continues the cache as if it had been decoded so."""
    g, rng = gen(50), random.Random(50)
    L, H, K, D, page, V, B, hidden = 2, 8, 2, 64, 16, 500, 3, 256
    w = [{n: randn(g, hidden, m * D, scale=hidden ** -0.5) for n, m in (("q", H), ("k", K), ("v", K))} | {"o": randn(g, H * D, hidden, scale=(H * D) ** -0.5)} for _ in range(L)]
    qw, kw = randn(g, D, scale=0.1) + 1, randn(g, D, scale=0.1) + 1
    embed, head, table = randn(g, V, hidden), randn(g, hidden, V, scale=0.4), rope_table(200, D)
    per = 10
    pages = torch.randperm(B * per, generator=g, device="cuda").int().view(B, per).contiguous()

    def fresh():
        return [tq.tq_kv_cache(*(torch.zeros(B * per, K, page, D, dtype=BF, device="cuda") for _ in range(2))) for _ in range(L)]

    def forward(caches, tokens, seq, position, state, first, lens, mask=None):
        """tokens [T] of sequences seq at their positions, kept at places state of the cache -> logits [T][V]"""
        slots = (pages[seq.long(), (state // page).long()] * page + state % page).int()
        h = embed[tokens.long()]
        for c, m in zip(caches, w):
            q = tq.tq_qk_norm_rope_append(h @ m["q"], h @ m["k"], h @ m["v"], qw, kw, table, position, slots, c)
            h = h + tq.tq_tree_attention(q, c, pages, first, lens, ws, mask=mask).float().flatten(1) @ m["o"]
        return h @ head

    settings = lambda n: dict(temperature=torch.full((n,), 0.8, device="cuda"), top_k=torch.full((n,), 20, dtype=torch.int32, device="cuda"),  # noqa: E731
                              top_p=torch.full((n,), 0.9, device="cuda"))
    prompt = [7, 20, 33]
    text = [[rng.randrange(V) for _ in range(n)] for n in prompt]

    def prefill(caches):
        flat = i32([t for x in text for t in x])
        pos = i32([i for n in prompt for i in range(n)])
        seq = i32([b for b, n in enumerate(prompt) for _ in range(n)])
        return forward(caches, flat, seq, pos, pos, i32([0, 7, 27, 60]), i32(prompt))

    # one by one: five steps, a uniform number for each place
    uniform = torch.rand(B, 64, generator=g, device="cuda")
    one, tree = fresh(), fresh()
    x = prefill(one)[[6, 26, 59]]
    token = tq.tq_sample(x, uniform[:, 0].contiguous(), **settings(B))
    steps, logits_one, lens = [token], [x], i32(prompt)
    for d in range(1, 6):
        lens = lens + 1
        x = forward(one, token, i32(range(B)), (lens - 1).int(), (lens - 1).int(), i32(range(B + 1)), lens)
        token = tq.tq_sample(x, uniform[:, d].contiguous(), **settings(B))
        steps.append(token), logits_one.append(x)
    # the same with drafts: right ones among wrong ones, in an order of their own; each sequence's right path ends elsewhere
    assert torch.equal(prefill(tree)[[6, 26, 59]], logits_one[0])
    right = [[int(s[b]) for s in steps] for b in range(B)]  # right[b][0] is certain, the others are to be found
    n, tokens, parents, depth, found = 12, [], [], [], [4, 1, 5]
    for b in range(B):
        par, tok, dep, at = [-1], [right[b][0]], [0], 0
        chain = [0]
        for i in range(1, n):
            if len(chain) < found[b] and i % 2 == 0:  # the next right one
                par.append(chain[-1]), tok.append(right[b][len(chain)])
                chain.append(i)
            else:
                p = rng.randrange(i)
                par.append(p), tok.append(V + 1)  # a token that is never drawn
            dep.append(dep[par[-1]] + 1)
        parents += par
        tokens += tok
        depth += dep
    bits = torch.zeros(B * n, n, dtype=torch.bool)
    for b in range(B):
        for i in range(n):
            r = b * n + i
            if i:
                bits[r] = bits[b * n + parents[r]]
            bits[r, i] = True
    first, seq = i32([0, n, 2 * n, 3 * n]), i32([b for b in range(B) for _ in range(n)])
    lens = i32([p + n for p in prompt])
    pos = i32([prompt[b] + depth[b * n + i] for b in range(B) for i in range(n)])
    state = i32([prompt[b] + i for b in range(B) for i in range(n)])
    x = forward(tree, i32(tokens).clamp(max=V - 1), seq, pos, state, first, lens, pack(bits, 1))
    u = uniform[seq.long(), (i32(depth) + 1).long()].contiguous()
    sampled = tq.tq_sample(x, u, **settings(B * n))
    out, path, count, after = tq.tq_tree_accept(tq.tq_kv_caches(tree), pages, first, lens, i32(tokens), i32(parents), sampled, 8)
    assert count.tolist() == found
    for b in range(B):
        assert out[b, :found[b]].tolist() == right[b][1:found[b] + 1]
        for d in range(found[b]):
            a, e = x[b * n + int(path[b, d])], logits_one[d + 1][b]
            # the two ways differ by roundings to bf16 alone: queries, keys, values and outputs in two layers, 2^-8 each of numbers of order 1
            assert float((a - e).abs().max()) <= 16 * HALF * float(e.abs().max())
        assert after[b] == prompt[b] + found[b]
        for c, e in zip(tree, one):
            for s in range(int(after[b])):
                at = (int(pages[b, s // page]), slice(None), s % page)
                for got, ref in ((c.k, e.k), (c.v, e.v)):
                    assert float((got[at].float() - ref[at].float()).abs().max()) <= 8 * HALF * float(ref[at].float().abs().max()) + 1e-6
    assert all(tq.tq_kv_cache_status(c) == 0 for c in one + tree)


# ------------------------------------------------------------------------------------------------ the binding
def test_refusals_of_the_binding(tq, ws):
    g = gen(60)
    kp = randn(g, 4, 2, 16, 64, dtype=BF)
    c = tq.tq_kv_cache(kp, kp.clone())
    q, u, x = randn(g, 3, 4, 64, dtype=BF), torch.rand(3, device="cuda"), randn(g, 3, 50)
    table, first, lens = i32([[0, 1]]), i32([0, 3]), i32([9])
    bad = [
        lambda: tq.tq_tree_attention(q.float(), c, table, first, lens, ws), lambda: tq.tq_tree_attention(q.cpu(), c, table, first, lens, ws),
        lambda: tq.tq_tree_attention(q, c, table, first[:1], lens, ws), lambda: tq.tq_tree_attention(q, c, table, first.long(), lens, ws),
        lambda: tq.tq_tree_attention(q, c, table, first, lens.cpu(), ws), lambda: tq.tq_tree_attention(q, c, table.t(), first, lens, ws),
        lambda: tq.tq_tree_attention(q, c, table, first, lens, ws, mask=i32([[1]])), lambda: tq.tq_tree_attention(q, c, table, first, lens, ws, mask=i32([[1]] * 3).bool()),
        lambda: tq.tq_tree_attention(q, c, table, first, lens, ws, out=torch.empty(3, 4, 64, device="cuda")),
        lambda: tq.tq_tree_attention(q, c, table, first, lens, ws, lse=torch.empty(3, device="cuda")),
        lambda: tq.tq_sample(x.double(), u), lambda: tq.tq_sample(x, u[:2]), lambda: tq.tq_sample(x, u.double()), lambda: tq.tq_sample(x.t().contiguous().t(), u),
        lambda: tq.tq_sample(x, u, top_k=u), lambda: tq.tq_sample(x, u, top_p=i32([1, 1, 1])), lambda: tq.tq_sample(x, u, temperature=u.cpu()),
        lambda: tq.tq_sample(x, u, out=torch.empty(3, dtype=torch.int64, device="cuda")), lambda: tq.tq_sample(x, u, logprob=i32([1, 1, 1])),
        lambda: tq.tq_tree_accept(tq.tq_kv_caches([c]), None, first, lens, i32([1] * 3), i32([0] * 3), i32([1] * 3), 4),
        lambda: tq.tq_tree_accept(None, None, first, lens, i32([1] * 3), i32([0] * 2), i32([1] * 3), 4),
        lambda: tq.tq_tree_accept(None, None, first, lens, i32([1] * 3), i32([0] * 3), i32([1] * 3), 0),
        lambda: tq.tq_qk_norm_rope_append(q, kp[:3, :, 0], kp[:3, :, 0], u, torch.ones(64, device="cuda"), rope_table(8, 64), i32([0] * 3), i32([0] * 3), c),
    ]
    for n, call in enumerate(bad):
        with pytest.raises((AssertionError, AttributeError)):
            call()
            pytest.fail(f"call {n} was not refused")
    with pytest.raises(tq.TqError):
        tq.tq_tree_attention(q, c, table, first, lens, ws, scale=0.0)
    with pytest.raises(tq.TqError):
        tq.tq_tree_accept(None, None, first, lens, i32([1] * 3), i32([0] * 3), i32([1] * 3), tq.TQ_TREE_MAX_PATH + 1)


def test_native_and_python_form_of_a_call_agree(tq, ws, monkeypatch):
    """The usual calls are served by the native module (none of them falls through it), and the Python form gives the same bits."""
    g = gen(61)
    c = tq.tq_kv_cache(randn(g, 9, 2, 16, 64, dtype=BF), randn(g, 9, 2, 16, 64, dtype=BF))
    q, k, v = randn(g, 6, 4 * 64), randn(g, 6, 2, 64), randn(g, 6, 2 * 64 + 8)[:, :128]
    w, rope, pos, slots = torch.rand(64, generator=g, device="cuda"), rope_table(20, 64), i32([[3, 4, 5, 6, 7, 8]] * 2), i32([0, 1, 2, 40, 41, -1])
    table, first, lens, mask = i32([[0, 1, 2], [5, 6, 7]]), i32([0, 4, 6]), i32([40, 20]), i32([[1], [3], [1], [7], [1], [3]])
    x, u, t, p = randn(g, 6, 3000, scale=3), torch.rand(6, generator=g, device="cuda"), f32([0.7] * 6), f32([0.9] * 6)
    tokens, parents, sampled = i32([1, 2, 3, 4, 5, 6]), i32([-1, 0, 1, 0, -1, 0]), i32([2, 3, 4, 4, 6, 6])
    caches = tq.tq_kv_caches([c])

    def calls():
        qb = torch.randn(6, 4, 64, generator=gen(62), device="cuda").to(BF)
        lse = torch.empty(6, 4, device="cuda")
        yield tq.tq_qk_norm_rope_append(q, k, v, w, w, rope, pos, slots, c, sections=(20, 12), interleaved=True)
        yield tq.tq_qk_norm_rope_append(q, k, v, w, w, rope, pos[0], slots, c, eps=1e-6, out=torch.empty(6, 4, 64, dtype=BF, device="cuda"))
        yield tq.tq_tree_attention(qb, c, table, first, lens, ws, mask=mask, lse=lse)
        yield lse
        yield tq.tq_tree_attention(qb, c, table, first, lens, ws, scale=0.3, out=torch.empty_like(qb))
        yield tq.tq_sample(x, u)
        yield from tq.tq_sample(x.to(BF), u, temperature=t, top_p=p, min_p=t * 0.01, logprob=True)
        yield from tq.tq_tree_accept(caches, table, first, lens, tokens, parents, sampled, 3)
        yield from tq.tq_tree_accept(None, None, first, lens, tokens, parents, sampled, 5)

    if tq._fast is None:
        pytest.skip("the native module is not here")
    k0, v0 = c.k.clone(), c.v.clone()
    with monkeypatch.context() as m:
        m.setattr(tq, "_check", lambda rc, name: pytest.fail(f"{name} was not served by the native module"))
        native = [y.clone() for y in calls()]
    k1, v1 = c.k.clone(), c.v.clone()
    c.k.copy_(k0), c.v.copy_(v0)
    monkeypatch.setattr(tq, "_fast", None)
    python = list(calls())
    assert all(torch.equal(a, b) for a, b in zip(native, python)) and torch.equal(c.k, k1) and torch.equal(c.v, v1)


def test_weights_of_any_alignment(tq):
    g = gen(63)
    kp = randn(g, 2, 2, 16, 128, dtype=BF)
    c = tq.tq_kv_cache(kp, kp.clone())
    q, k, w = randn(g, 3, 4, 128), randn(g, 3, 2, 128), randn(g, 260)
    args = (rope_table(9, 128), i32([1, 2, 3]), i32([3, 4, 5]), c)
    for at in (0, 1, 3, 4):
        want = tq.tq_qk_norm_rope_append(q, k, k, w[at:at + 128].clone(), w[at + 128:at + 256].clone(), *args)
        kw = kp.clone()
        assert torch.equal(tq.tq_qk_norm_rope_append(q, k, k, w[at:at + 128], w[at + 128:at + 256], *args), want) and torch.equal(kp, kw)


def test_a_pool_that_is_given_twice_is_moved_once(tq):
    """A path on which every state comes from where an earlier one's neighbour lay: moved twice at once, states would be lost."""
    g, n, K, D, page = gen(78), 40, 8, 128, 16
    kp, vp = randn(g, 8, K, page, D, dtype=BF), randn(g, 8, K, page, D, dtype=BF)
    table, length = torch.randperm(8, generator=g, device="cuda").int()[None].contiguous(), 100
    path = [0] + list(range(2, n))  # row 1 is not taken
    parents, tokens = [-1, 0, 0] + list(range(2, n - 1)), [5, 1] + [2 + i % 3 for i in range(n - 2)]
    sampled = [tokens[2], 0] + [tokens[i + 1] for i in range(2, n - 1)] + [9]
    place = table[0].long()
    want = [x[place].transpose(1, 2).reshape(-1, K, D).clone() for x in (kp, vp)]
    for w in want:
        w[length - n:length - n + len(path)] = w[[length - n + i for i in path]]
    c = tq.tq_kv_cache(kp, vp)
    caches = tq.tq_kv_caches([c, tq.tq_kv_cache(vp, kp), c, tq.tq_kv_cache(kp, kp)] * 8)
    got = tq.tq_tree_accept(caches, table, i32([0, n]), i32([length]), i32(tokens), i32(parents), i32(sampled), n)
    assert got[1].tolist() == [path + [-1]] and got[2].tolist() == [n - 1] and got[3].tolist() == [length - 1]
    for x, w in zip((kp, vp), want):
        assert torch.equal(x[place].transpose(1, 2).reshape(-1, K, D)[:length - 1], w[:length - 1])


def test_a_spoiled_row_of_a_long_cache(tq, ws):
    """An infinite value that the others do not see, behind a cache of many tiles in several CTAs: they are computed again from what they see."""
    g, n, H, K, D, page, length = gen(77), 20, 8, 1, 128, 16, 9001
    P = -(-length // page)
    kp, vp = randn(g, P, K, page, D, dtype=BF), randn(g, P, K, page, D, dtype=BF)
    q, table = randn(g, n, H, D, dtype=BF, scale=1.5), torch.randperm(P, generator=g, device="cuda").int()[None].contiguous()
    bits = torch.eye(n, dtype=torch.bool)
    bits[:, 0] = True
    k, v = (x[table[0].long(), 0].reshape(-1, D)[:length].clone() for x in (kp, vp))
    s = length - n + 7
    vp[int(table[0, s // page]), 0, s % page] = -INF
    out, lse = torch.empty(n, H, D, dtype=BF, device="cuda"), torch.empty(n, H, device="cuda")
    tq.tq_tree_attention(q, tq.tq_kv_cache(kp, vp), table, i32([0, n]), i32([length]), ws, mask=pack(bits, 1), out=out, lse=lse)
    seen = torch.ones(n, length, dtype=torch.bool, device="cuda")
    seen[:, length - n:] = bits.cuda()
    others = [i for i in range(n) if i != 7]
    for h in range(H):
        want, wl, bound = attend_ref(q[others, h], k, v, seen[others], D ** -0.5)
        within(out[others, h], want, bound)
        check_lse(lse[others, h], wl)
    assert bool((out[7] == -INF).all())
