"""The operators between the linear layers against their formulas in 64 bits.

Where the bounds come from.  A bf16 result is one rounding to nearest: 2^-8 of its value (HALF).  Norm: the sum of up to
16384 squares runs through at most 32 + 10 fp32 additions, so 1/rms is within 42/2 * 2^-24 < 2^-18 with its root and
division.  Rotation: two products and a sum in fp32, within 2^-22 of |a| + |b|, with table values taken as given.
Attention: p is rounded to bf16 (2^-8 of itself) before the product with v, and its exponent carries the fp32 error of
a dot product of up to 128 terms (128 * 2^-24 * sum |q k| scale, below 2^-11 for the sums of up to 60 here) and of
exp2 (2^-22): out is within (2^-8 + 2^-10) * sum p |v| / sum p of the formula, before its own rounding."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
HALF = 2.0 ** -8  # half the spacing of bf16's 8 significant bits, relative


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


def within(got, ref, bound):
    err = (got.to(F64) - ref).abs()
    assert bool((err <= bound).all()), (float((err - bound).max()), float(err.max()))


# ------------------------------------------------------------------------------------------------ norm
def norm_ref(h, w, d, eps):
    x = h.to(F64) + (0 if d is None else d.to(F64))
    return x, x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.to(F64)


SHAPES = [(1, 1), (1, 7), (3, 64), (5, 128), (17, 120), (9, 130), (2, 256), (6, 248), (4, 1000), (1, 2048), (1, 8192), (3, 5001), (2, 16384), (1, 16383),
          (601, 128), (600, 768), (599, 4104), (400, 4097), (300, 16384)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("ht,dt", [(BF, None), (BF, F32), (BF, BF), (F32, None), (F32, F32), (F32, BF)])
def test_rmsnorm(tq, rows, cols, ht, dt):
    g = gen(rows * 31 + cols)
    h, w = randn(g, rows, cols, dtype=ht, scale=3), randn(g, cols, scale=0.2) + 1
    d = None if dt is None else randn(g, rows, cols, dtype=dt)
    x, n = norm_ref(h, w, d, 1e-5)
    ho = torch.full_like(h, float("nan"))
    before = h.clone()
    out = tq.tq_rmsnorm(h, w, d, eps=1e-5, h_out=ho)
    assert torch.equal(h, before)
    within(out, n, n.abs() * (HALF + 2.0 ** -17) + 1e-30)
    within(ho, x, x.abs() * (HALF if ht == BF else 2.0 ** -24))
    if dt is not None:  # in place
        inplace = h.clone()
        assert torch.equal(tq.tq_rmsnorm(inplace, w, d, eps=1e-5), out) and torch.equal(inplace, ho)
    q, s = tq.tq_rmsnorm_q8(h, w, d, eps=1e-5, h_out=ho)
    top = n.abs().amax(-1)
    within(s, torch.where(top > 0, top / 127, 1.0), top / 127 * 2.0 ** -17)
    step = s.to(F64)[:, None]
    within(q.to(F64) * step, n, 0.5 * step * (1 + 2.0 ** -9) + n.abs() * 2.0 ** -17)
    assert int(q.abs().max()) <= 127 and bool((q.abs().amax(-1) == 127).all())
    within(ho, x, x.abs() * (HALF if ht == BF else 2.0 ** -24))


def test_rmsnorm_strides_and_unaligned_rows(tq):
    g = gen(5)
    for rows, cols, pitch, at in [(7, 256, 264, 8), (7, 256, 257, 0), (7, 256, 264, 3), (700, 512, 520, 1), (40, 128, 640, 128)]:
        base, db = randn(g, rows * pitch + at, dtype=BF, scale=2), randn(g, rows * (pitch + 8) + at)
        h = base[at:].as_strided((rows, cols), (pitch, 1), at)
        d = db.as_strided((rows, cols), (pitch + 8, 1), at)
        w = randn(g, cols + 1)[1:]
        x, n = norm_ref(h, w, d, 1e-6)
        copy = base.clone()
        out = tq.tq_rmsnorm(h, w, d, eps=1e-6)
        within(out, n, n.abs() * (HALF + 2.0 ** -17) + 1e-30)
        within(h, x, x.abs() * HALF)
        touched = torch.zeros_like(base, dtype=torch.bool)
        touched.as_strided((rows, cols), (pitch, 1), at).fill_(True)
        assert torch.equal(base[~touched], copy[~touched])  # nothing beside the rows was written


def test_rmsnorm_zero_and_non_finite_rows(tq):
    g = gen(6)
    h, w = randn(g, 6, 512), randn(g, 512)
    h[1] = 0
    h[2, 17] = float("nan")
    h[3, 400] = float("inf")
    _, n = norm_ref(h, w, None, 1e-5)
    out = tq.tq_rmsnorm(h, w, eps=1e-5)
    q, s = tq.tq_rmsnorm_q8(h, w, eps=1e-5)
    for r in (0, 4, 5):
        within(out[r], n[r], n[r].abs() * (HALF + 2.0 ** -17) + 1e-30)
    assert not out[1].any() and not q[1].any() and float(s[1]) == 1.0
    assert bool(out[2].isnan().all()) and bool(s[2].isnan()) and not q[2].any()
    assert bool(out[3, 400].isnan()) and not out[3, :400].any() and bool(s[3].isnan()) and not q[3].any()
    z = torch.zeros(2, 64, device="cuda", dtype=BF)
    assert bool(tq.tq_rmsnorm(z, torch.ones(64, device="cuda"), eps=0.0).isnan().all())  # 0 / 0 when eps is 0
    assert tq.tq_rmsnorm(h[:0], w).shape == (0, 512)


# ------------------------------------------------------------------------------------------------ rotary positions, cache write
def rope_table(n, rot):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=F64, device="cuda") / rot)
    a = torch.arange(n, dtype=F64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def rope_ref(x, table, positions, sections, interleaved):
    """x [T][n][D]; -> (rotated, sum of the magnitudes that went into each element)"""
    x = x.to(F64)
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
def test_rope_append(tq, H, K, D, rot, interleaved, xt, T, axes):
    g = gen(T + H + rot)
    page = 24
    sections = {1: [rot // 2], 2: [rot // 2 - 3, 3], 3: [1, rot // 2 - 1, 0]}[axes]
    pages = T // page + 3
    kp, vp = randn(g, pages, K, page, D, dtype=BF), randn(g, pages, page, K, D, dtype=BF).transpose(1, 2)
    vp = vp.contiguous() if T % 2 else vp  # both pools have one layout; it alternates between the cases
    kp = kp if T % 2 else kp.transpose(1, 2).contiguous().transpose(1, 2)
    cache = tq.tq_kv_cache(kp, vp)
    wide = randn(g, T, (H + 2 * K) * D + 8, dtype=xt)  # q, k, v side by side, as one product leaves them
    q, k, v = wide[:, :H * D], wide[:, H * D:(H + K) * D], wide[:, (H + K) * D:(H + 2 * K) * D]
    table = rope_table(500, rot)
    pos = torch.randint(0, 500, (axes, T), generator=g, device="cuda", dtype=torch.int32)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T].int()
    slots[T // 2] = -1
    want_k, want_v = kp.to(F64).clone(), vp.to(F64).clone()
    keep = slots >= 0
    at = slots[keep].long()
    rk, mk = rope_ref(k.reshape(T, K, D), table, pos, sections, interleaved)
    bound_k = torch.zeros_like(want_k)
    want_k[at // page, :, at % page] = rk[keep]
    bound_k[at // page, :, at % page] = rk[keep].abs() * HALF + mk[keep] * 2.0 ** -21
    want_v[at // page, :, at % page] = v.reshape(T, K, D)[keep].to(BF).to(F64)
    out = tq.tq_rope_append(q, k, v, table, pos, slots, cache, sections=sections, interleaved=interleaved)
    rq, mq = rope_ref(q.reshape(T, H, D), table, pos, sections, interleaved)
    within(out, rq, rq.abs() * HALF + mq * 2.0 ** -21)
    within(kp, want_k, bound_k)
    assert torch.equal(vp.to(F64), want_v)
    assert tq.tq_kv_cache_status(cache) == 0


def test_rope_append_keeps_off_what_is_out_of_range(tq):
    g = gen(9)
    kp, vp = randn(g, 2, 2, 16, 64, dtype=BF), randn(g, 2, 2, 16, 64, dtype=BF)
    k0, v0 = kp.clone(), vp.clone()
    cache = tq.tq_kv_cache(kp, vp)
    q, k, v = randn(g, 4, 4, 64), randn(g, 4, 2, 64), randn(g, 4, 2, 64)
    table = rope_table(10, 64)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = tq.tq_rope_append(q, k, v, table, i32(0, 10, -1, 9), i32(-1, 1, 2, -1), cache)
    assert tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_POSITION
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    assert bool(out[1:3].isnan().all()) and not bool(out[0].isnan().any()) and not bool(out[3].isnan().any())
    out = tq.tq_rope_append(q, k, v, table, i32(1, 2, 3, 4), i32(32, 31, -2, 2 ** 31 - 1), cache)
    assert tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_PAGE  # slots below 0 are padding
    assert torch.equal(vp[1, :, 15], v[1].to(BF)) and int((vp != v0).sum()) <= 2 * 64 and bool(out.isfinite().all())
    assert tq.tq_kv_cache_status(cache) == 0
    assert tq.tq_rope_append(q[:0], k[:0], v[:0], table, i32(), i32(), cache).shape == (0, 4, 64)


# ------------------------------------------------------------------------------------------------ attention
def attend_ref(q, k, v, seen, scale):
    """q [n][D], k / v [m][D], seen [n][m] -> out, lse, bound of out; what is not seen is not touched."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    x = torch.where(seen, q @ torch.where(seen.any(0)[:, None], k, 0.0).t() * scale, -math.inf)
    lse = torch.logsumexp(x, -1) if x.shape[1] else torch.full((q.shape[0],), -math.inf, dtype=F64, device=q.device)
    p = torch.where(seen, torch.exp(x - torch.where(lse.isfinite(), lse, 0.0)[:, None]), 0.0)
    vs = torch.where(seen.any(0)[:, None], v, 0.0)
    out = p @ vs
    return out, lse, (p @ vs.abs()) * (HALF + 2.0 ** -10) + out.abs() * HALF + 1e-30


def check_lse(got, want):
    empty = want == -math.inf
    assert torch.equal(got == -math.inf, empty)
    within(got[~empty], want[~empty], 2.0 ** -11 + want[~empty].abs() * 2.0 ** -20)


def paged_case(tq, ws, lens, H, K, D, page, seed, layout=0, max_pages=None, spoil=True):
    g = gen(seed)
    B = len(lens)
    need = [-(-max(n, 0) // page) for n in lens]
    pool = sum(need) + 2
    shape = (pool, K, page, D) if layout == 0 else (pool, page, K, D)
    kp, vp = randn(g, *shape, dtype=BF), randn(g, *shape, dtype=BF)
    if layout:
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    perm = torch.randperm(pool, generator=g, device="cuda")
    cols = max(max(need), 1) if max_pages is None else max_pages
    table = torch.full((B, cols), -7, dtype=torch.int32, device="cuda")  # entries past a length are not followed
    at = 0
    used = torch.zeros(pool, page, dtype=torch.bool, device="cuda")
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n].int()
        if lens[b] > 0:
            flat = torch.arange(n * page, device="cuda") < lens[b]
            used[perm[at:at + n]] = flat.view(n, page)
        at += n
    if spoil:  # slots that no length reaches hold NaN and infinities
        kp.masked_fill_(~used[:, None, :, None], float("nan"))
        vp.masked_fill_(~used[:, None, :, None], float("inf"))
    q = randn(g, B, H, D, dtype=BF, scale=1.5)
    cache = tq.tq_kv_cache(kp, vp)
    lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    lse = torch.full((B, H), float("nan"), device="cuda")
    out = tq.tq_paged_attention(q, cache, table, lt, ws, lse=lse)
    again = tq.tq_paged_attention(q, cache, table, lt, ws)
    assert torch.equal(out, again)  # the same call, the same bits
    at = 0
    for b, n in enumerate(need):
        ids = perm[at:at + n]
        at += n
        for h in range(K):
            k, v = (x[ids, h].reshape(-1, D)[:max(lens[b], 0)] for x in (kp, vp))
            hs = slice(h * (H // K), (h + 1) * (H // K))
            seen = torch.ones(H // K, k.shape[0], dtype=torch.bool, device="cuda")
            want, wl, bound = attend_ref(q[b, hs], k, v, seen, D ** -0.5)
            within(out[b, hs], want, bound)
            check_lse(lse[b, hs], wl)
    assert tq.tq_kv_cache_status(cache) == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,K", [(4, 4), (6, 2), (8, 1), (24, 8), (20, 2), (16, 1)])
@pytest.mark.parametrize("lens,page", [([1], 16), ([37], 16), ([64, 0, 65, 1], 1), ([500, 15, 16, 17, 129], 24), ([0, 0], 8), ([3000, -3, 77], 64)])
def test_paged_attention(tq, ws, D, H, K, lens, page):
    paged_case(tq, ws, lens, H, K, D, page, seed=sum(lens) + H, layout=(H + page) % 2)


def test_paged_attention_many_sequences(tq, ws):
    g = gen(3)
    lens = torch.randint(0, 400, (700,), generator=g, device="cuda").tolist()
    paged_case(tq, ws, lens, 4, 2, 64, 16, seed=11)


def test_paged_attention_long(tq, ws):
    paged_case(tq, ws, [100003, 5], 8, 2, 128, 48, seed=12)


def test_paged_attention_large_scores(tq, ws):
    """Scores of several hundred: one state takes all the weight, whatever came before it in the running maximum."""
    g = gen(13)
    kp, vp = randn(g, 8, 1, 32, 64, dtype=BF), randn(g, 8, 1, 32, 64, dtype=BF)
    q = randn(g, 1, 2, 64, dtype=BF)
    kp[3, 0, 7] = q[0, 0] * 60
    kp[6, 0, 1] = q[0, 0] * 70
    kp[5, 0, 9] = q[0, 1] * -80
    table = torch.arange(8, device="cuda", dtype=torch.int32)[None].contiguous()
    out = tq.tq_paged_attention(q, tq.tq_kv_cache(kp, vp), table, torch.tensor([256], dtype=torch.int32, device="cuda"), ws)
    k, v = kp.flatten(0, 2), vp.flatten(0, 2)
    x = q[0].to(F64) @ k.to(F64).t() / 8
    w = torch.softmax(x, 1)
    assert float(x.max()) > 400 and float(w[0].max()) > 0.999
    # the exponent's error grows with the score: 2^-24 * 64 * sum |q k| / 8, below 2^-7 here
    within(out[0], w @ v.to(F64), (w @ v.to(F64).abs()) * (HALF + 2.0 ** -6) + 2.0 ** -8)


def test_paged_attention_refuses_pages_and_lengths_out_of_range(tq, ws):
    g = gen(14)
    kp, vp = randn(g, 3, 1, 16, 64, dtype=BF), randn(g, 3, 1, 16, 64, dtype=BF)
    cache, q = tq.tq_kv_cache(kp, vp), randn(g, 2, 2, 64, dtype=BF)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = tq.tq_paged_attention(q, cache, i32([[0, 3], [1, -1]]), i32([32, 20]), ws)
    assert tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_PAGE
    ok = tq.tq_paged_attention(q, cache, i32([[0], [1]]), i32([16, 16]), ws)
    assert tq.tq_kv_cache_status(cache) == 0
    assert torch.equal(out, ok)  # a page outside the pool hides its states
    cut = tq.tq_paged_attention(q, cache, i32([[0], [1]]), i32([17, 2 ** 31 - 1]), ws)
    assert tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_PAGE and torch.equal(cut, ok)
    assert tq.tq_paged_attention(q[:0], cache, i32([[0]])[:0], i32([]), ws).shape == (0, 2, 64)


def test_paged_attention_propagates_what_is_visible(tq, ws):
    g = gen(15)
    kp, vp = randn(g, 2, 1, 16, 64, dtype=BF), randn(g, 2, 1, 16, 64, dtype=BF)
    kp[1, 0, 3, 5] = float("nan")
    vp[0, 0, 2, 9] = float("inf")
    q = randn(g, 2, 1, 64, dtype=BF)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = tq.tq_paged_attention(q, tq.tq_kv_cache(kp, vp), i32([[0], [1]]), i32([16, 16]), ws)
    assert bool(out[1].isnan().all()) and float(out[0, 0, 9]) == math.inf and int(out[0].isfinite().sum()) == 63


def cross_case(tq, ws, B, T, S, H, K, D, kv_len=None, block=0, seed=0, mask_rate=0.5, spoil=True, expand=False, layout=0):
    g = gen(seed + T * 7 + S)
    pad = 8 * D
    qf = randn(g, B, T, H * D + pad, dtype=BF, scale=1.5)
    q = qf[..., :H * D].unflatten(-1, (H, D))
    shape = (1 if expand else B, S, K, D) if layout == 0 else (1 if expand else B, K, S, D)
    k, v = randn(g, *shape, dtype=BF), randn(g, *shape, dtype=BF)
    if layout:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    mask = None
    seen = torch.ones(B, T, S, dtype=torch.bool, device="cuda")
    if block:
        n = -(-S // block)
        mask = torch.rand(B, T, n, generator=g, device="cuda") < mask_rate
        mask[0, T // 2] = False  # a token that sees nothing
        seen &= mask.repeat_interleave(block, -1)[..., :S]
    kl = None
    if kv_len is not None:
        kl = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
        seen &= torch.arange(S, device="cuda") < kl[:, None, None].clamp(0, S)
    if spoil and not expand:  # states that no token of the sequence sees
        hidden = ~seen.any(1)
        k.masked_fill_(hidden[:, :, None, None], float("nan"))
        v.masked_fill_(hidden[:, :, None, None], float("nan"))
        if B * T > 1 and block and bool(seen.any()):  # and a state that one token sees and the others do not
            b, t, s = (int(i) for i in torch.nonzero(seen)[seen.sum() // 2])
            only = seen.clone()
            seen_elsewhere = only[b, :, s].clone()
            seen_elsewhere[t] = False
            if bool((~only[b, :, s]).any()):
                v[b, s] = float("inf")
    if expand:
        k, v = k.expand(B, -1, -1, -1), v.expand(B, -1, -1, -1)
    lse = torch.full((B, T, H), float("nan"), device="cuda")
    out = tq.tq_cross_attention(q, k, v, ws, kv_len=kl, mask=mask, block_len=block, lse=lse)
    assert torch.equal(out.nan_to_num(7.0), tq.tq_cross_attention(q, k, v, ws, kv_len=kl, mask=mask, block_len=block).nan_to_num(7.0))
    for b in range(B):
        for h in range(K):
            for i in range(h * (H // K), (h + 1) * (H // K)):
                bad = v[b, :, h].isinf().any(-1)
                clean_v = torch.where(bad[:, None], 0.0, v[b, :, h].to(F64)) if spoil else v[b, :, h]
                want, wl, bound = attend_ref(q[b, :, i], k[b, :, h], clean_v, seen[b], D ** -0.5)
                hit = seen[b][:, bad].any(-1)  # tokens that do see an infinite value
                assert not bool(out[b, hit, i].isfinite().any())
                within(out[b, ~hit, i], want[~hit], bound[~hit])
                check_lse(lse[b, :, i], wl)
    assert tq.tq_attn_status(ws) == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,S,H,K", [(1, 1, 1, 2, 1), (2, 1, 1601, 8, 2), (1, 2, 64, 4, 4), (2, 3, 65, 6, 2), (1, 17, 200, 16, 2), (2, 70, 333, 8, 2),
                                       (1, 129, 130, 20, 2), (1, 300, 1000, 3, 1), (3, 33, 128, 9, 9)])
def test_cross_attention(tq, ws, D, B, T, S, H, K):
    cross_case(tq, ws, B, T, S, H, K, D, layout=S % 2)


@pytest.mark.parametrize("T", [1, 2, 65, 130])
@pytest.mark.parametrize("S,block", [(200, 1), (300, 7), (500, 100), (640, 128), (1000, 1000), (1300, 333), (90, 500)])
def test_cross_attention_masks(tq, ws, T, S, block):
    cross_case(tq, ws, 2, T, S, 8, 2, 128, kv_len=[S, max(1, S // 2 + 3)], block=block, seed=1)
    cross_case(tq, ws, 2, T, S, 4, 4, 64, block=block, seed=2, mask_rate=0.1, layout=1)


@pytest.mark.parametrize("T", [1, 3, 140])
def test_cross_attention_lengths(tq, ws, T):
    cross_case(tq, ws, 4, T, 300, 8, 4, 64, kv_len=[0, 1, 300, 129], seed=3)
    cross_case(tq, ws, 3, T, 257, 4, 1, 128, kv_len=[-4, 256, 1000], seed=4, spoil=False)
    cross_case(tq, ws, 1, T, 0, 4, 2, 128, seed=5)


@pytest.mark.parametrize("T", [1, 40])
def test_cross_attention_shared_states(tq, ws, T):
    cross_case(tq, ws, 3, T, 500, 8, 2, 128, kv_len=[500, 77, 300], seed=6, expand=True)


def test_cross_attention_split_over_the_states(tq, ws):
    cross_case(tq, ws, 1, 5, 20000, 8, 1, 128, seed=7)
    cross_case(tq, ws, 1, 1, 30001, 8, 2, 64, seed=8, block=2000)
    cross_case(tq, ws, 1, 130, 9000, 2, 1, 64, seed=9, block=601)


def test_cross_attention_many_groups_of_different_lengths(tq, ws):
    """More groups than the workspace can number, of lengths that make cutting them worth while."""
    cross_case(tq, ws, 9, 20, 1500, 64, 64, 64, kv_len=[1500, 3, 700, 1500, 1100, 0, 900, 1499, 128], seed=10)


@pytest.mark.parametrize("T", [1, 40])
def test_cross_attention_one_head_for_all(tq, ws, T):
    """Keys and values whose heads are one head, expanded (stride 0)."""
    g = gen(23)
    q, k, v = randn(g, 2, T, 8, 64, dtype=BF), randn(g, 2, 300, 1, 64, dtype=BF), randn(g, 2, 300, 1, 64, dtype=BF)
    wide = tq.tq_cross_attention(q, k.expand(-1, -1, 4, -1), v.expand(-1, -1, 4, -1), ws)
    assert torch.equal(wide, tq.tq_cross_attention(q, k.repeat(1, 1, 4, 1), v.repeat(1, 1, 4, 1), ws))


@pytest.mark.parametrize("T", [1, 50])
def test_cross_attention_large_scores(tq, ws, T):
    """A maximum that keeps rising along the states: the running results are rescaled again and again."""
    g = gen(16)
    S, D = 2000, 64
    q = randn(g, 1, T, 2, D, dtype=BF)
    k, v = randn(g, 1, S, 1, D, dtype=BF, scale=0.1), randn(g, 1, S, 1, D, dtype=BF)
    k += (q[:, :1, :1].float() * torch.linspace(0, 12, S, device="cuda")[None, :, None, None]).to(BF)
    out = tq.tq_cross_attention(q, k, v, ws)
    x = q[0].to(F64).flatten(0, 1) @ k[0, :, 0].to(F64).t() / 8
    w = torch.softmax(x, 1)
    assert float(x[0].max()) > 70
    # as above, with sum |q k| / 8 up to 250 in the exponent
    within(out[0].flatten(0, 1), w @ v[0, :, 0].to(F64), (w @ v[0, :, 0].to(F64).abs()) * (HALF + 2.0 ** -8) + 2.0 ** -9 * 4)


def test_cross_attention_keeps_a_broken_query_to_itself(tq, ws):
    g = gen(17)
    q, k, v = randn(g, 1, 9, 4, 64, dtype=BF), randn(g, 1, 300, 2, 64, dtype=BF), randn(g, 1, 300, 2, 64, dtype=BF)
    good = tq.tq_cross_attention(q, k, v, ws)
    q[0, 4, 1, 3] = float("nan")
    out = tq.tq_cross_attention(q, k, v, ws)
    assert bool(out[0, 4, 1].isnan().all())
    out[0, 4, 1] = good[0, 4, 1]
    assert torch.equal(out, good)


def test_offsets_past_32_bits(tq, ws):
    """A pool and encoder states whose elements lie more than 2^32 elements apart."""
    g = gen(18)
    far = 2 ** 31 + 64  # elements from page to page and from sequence to sequence
    buf = [torch.zeros(2 * far + 4096, dtype=BF, device="cuda") for _ in range(2)]
    kp, vp = (b.as_strided((3, 1, 16, 64), (far, 1024, 64, 1)) for b in buf)
    cache = tq.tq_kv_cache(kp, vp)
    q, k, v = randn(g, 32, 2, 64), randn(g, 32, 1, 64), randn(g, 32, 1, 64)
    slots = torch.arange(16, 48, device="cuda", dtype=torch.int32)  # pages 1 and 2
    table = rope_table(64, 64)
    pos = torch.arange(32, device="cuda", dtype=torch.int32)
    rot = tq.tq_rope_append(q, k, v, table, pos, slots, cache)
    want, mag = rope_ref(k, table, pos[None], [32], False)
    within(torch.cat([kp[1], kp[2]], 1).transpose(0, 1), want, want.abs() * HALF + mag * 2.0 ** -21)
    assert torch.equal(torch.cat([vp[1], vp[2]], 1).transpose(0, 1), v.to(BF))
    out = tq.tq_paged_attention(rot[-1:], cache, torch.tensor([[1, 2]], dtype=torch.int32, device="cuda"),
                                torch.tensor([32], dtype=torch.int32, device="cuda"), ws)
    seen = torch.ones(2, 32, dtype=torch.bool, device="cuda")
    keys, vals = torch.cat([kp[1, 0], kp[2, 0]]), torch.cat([vp[1, 0], vp[2, 0]])
    ref, _, bound = attend_ref(rot[-1], keys, vals, seen, 64 ** -0.5)
    within(out[0], ref, bound)
    ek, ev = (b.as_strided((3, 16, 1, 64), (far, 64, 64, 1)) for b in buf)
    for T in (1, 24):
        qq = randn(g, 3, T, 2, 64, dtype=BF)
        got = tq.tq_cross_attention(qq, ek, ev, ws)
        for h in range(2):
            ref, _, bound = attend_ref(qq[2, :, h], ek[2, :, 0], ev[2, :, 0], torch.ones(T, 16, dtype=torch.bool, device="cuda"), 64 ** -0.5)
            within(got[2, :, h], ref, bound)
    del buf, kp, vp, ek, ev, cache
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ streams, graphs
def test_streams_and_graphs(tq):
    g = gen(19)
    side = torch.cuda.Stream()
    w2 = tq.tq_attn_workspace(stream=side)
    h, wt, d = randn(g, 3, 256, dtype=BF), randn(g, 256), randn(g, 3, 256)
    q, k, v = randn(g, 3, 4, 64, dtype=BF), randn(g, 3, 200, 2, 64, dtype=BF), randn(g, 3, 200, 2, 64, dtype=BF)
    torch.cuda.synchronize()
    ref = tq.tq_rmsnorm(h, wt, d, h_out=torch.empty_like(h))
    torch.cuda.synchronize()
    out = tq.tq_rmsnorm(h, wt, d, h_out=torch.empty_like(h), stream=side)
    cross = tq.tq_cross_attention(q[:, None], k, v, w2, stream=side)
    side.synchronize()
    assert torch.equal(out, ref)
    ho, o1 = torch.empty_like(h), torch.empty(3, 256, dtype=BF, device="cuda")
    o2 = torch.empty(3, 1, 4, 64, dtype=BF, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tq.tq_rmsnorm(h, wt, d, h_out=ho, out=o1)
        tq.tq_cross_attention(q[:, None], k, v, w2, out=o2)
    for _ in range(3):
        o1.zero_(), o2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o1, ref) and torch.equal(o2, cross)
    assert tq.tq_attn_status(w2) == 0


def test_native_and_python_form_of_a_call_agree(tq, ws, monkeypatch):
    """The calls' usual case runs in a CPython module; the checks in Python make the same call of the library."""
    assert tq._fast is not None
    g = gen(20)
    h, w, d = randn(g, 5, 384, dtype=BF), randn(g, 384), randn(g, 5, 384)
    q, k, v = randn(g, 5, 6, 64), randn(g, 5, 2, 64), randn(g, 5, 2, 64)
    pos = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
    slots = torch.tensor([3, 17, -1, 30, 8], dtype=torch.int32, device="cuda")
    pages, lens = torch.tensor([[0, 1], [1, 0]], dtype=torch.int32, device="cuda"), torch.tensor([20, 9], dtype=torch.int32, device="cuda")
    enc, mask = randn(g, 2, 50, 2, 64, dtype=BF), torch.rand(2, 3, 5, generator=g, device="cuda") < 0.5
    table = rope_table(10, 64)
    base = randn(g, 2, 2, 16, 64, dtype=BF)

    def all_calls():
        kp, vp = base.clone(), base.clone()
        cache, ho = tq.tq_kv_cache(kp, vp), torch.empty_like(h)
        res = [tq.tq_rmsnorm(h, w), tq.tq_rmsnorm(h, w, d, h_out=ho), ho, *tq.tq_rmsnorm_q8(h, w, d, h_out=torch.empty_like(h))]
        res += [tq.tq_rope_append(q, k, v, table, pos, slots, cache, sections=[20, 12], interleaved=True), kp, vp]
        res += [tq.tq_rope_append(q.flatten(1), k, v, table, pos[1], slots, cache)]
        lse = torch.empty(2, 6, device="cuda")
        res += [tq.tq_paged_attention(res[-1][:2], cache, pages, lens, ws, lse=lse), lse]
        qq = randn(gen(21), 2, 3, 6, 64, dtype=BF)
        res += [tq.tq_cross_attention(qq, enc, enc, ws, kv_len=lens, mask=mask, block_len=10), tq.tq_cross_attention(qq[:, :1], enc, enc, ws, scale=0.3)]
        return res

    native = all_calls()
    monkeypatch.setattr(tq, "_fast", None)
    for a, b in zip(native, all_calls(), strict=True):
        assert a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b)


@pytest.mark.parametrize("native", [True, False])
def test_refusals_of_the_binding(tq, ws, monkeypatch, native):
    if not native:
        monkeypatch.setattr(tq, "_fast", None)
    g = gen(22)
    h, w = randn(g, 4, 64, dtype=BF), randn(g, 64)
    bad = (AssertionError, tq.TqError, KeyError, ValueError)
    for call in [lambda: tq.tq_rmsnorm(h.cpu(), w), lambda: tq.tq_rmsnorm(h.half(), w), lambda: tq.tq_rmsnorm(h, w[:63]), lambda: tq.tq_rmsnorm(h, w.to(BF)),
                 lambda: tq.tq_rmsnorm(h[0], w), lambda: tq.tq_rmsnorm(h.t(), w[:4]), lambda: tq.tq_rmsnorm(h, w, h[:3]), lambda: tq.tq_rmsnorm(h, w, h.half()),
                 lambda: tq.tq_rmsnorm(h, w, out=h.float()), lambda: tq.tq_rmsnorm(h, w, h, h_out=h.float()), lambda: tq.tq_rmsnorm(h, w, eps=-1.0)]:
        with pytest.raises(bad):
            call()
    kp = randn(g, 3, 2, 16, 64, dtype=BF)
    cache = tq.tq_kv_cache(kp, kp.clone())
    q, k, t, i = randn(g, 4, 4, 64), randn(g, 4, 2, 64), rope_table(9, 64), torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in [lambda: tq.tq_rope_append(q, k, q, t, i, i, cache), lambda: tq.tq_rope_append(q, k, k.to(BF), t, i, i, cache),
                 lambda: tq.tq_rope_append(q, k, k, t, i.long(), i, cache), lambda: tq.tq_rope_append(q, k, k, t, i, i[:3], cache),
                 lambda: tq.tq_rope_append(q, k, k, t, i, i, cache, sections=[31]), lambda: tq.tq_rope_append(q, k, k, t, i, i, cache, sections=[16, 16]),
                 lambda: tq.tq_rope_append(q, k, k, t[:, :60], i, i, cache), lambda: tq.tq_kv_cache(kp, kp[:2]), lambda: tq.tq_kv_cache(kp, kp.float())]:
        with pytest.raises(bad):
            call()
    qb, pages, lens = q.to(BF), torch.zeros(4, 2, dtype=torch.int32, device="cuda"), i
    for call in [lambda: tq.tq_paged_attention(q, cache, pages, lens, ws), lambda: tq.tq_paged_attention(qb[:, :3], cache, pages, lens, ws),
                 lambda: tq.tq_paged_attention(qb, cache, pages[:3], lens, ws), lambda: tq.tq_paged_attention(qb, cache, pages, lens.long(), ws),
                 lambda: tq.tq_paged_attention(qb, cache, pages, lens, ws, scale=0.0), lambda: tq.tq_paged_attention(qb, cache, pages, lens, ws, lse=lens)]:
        with pytest.raises(bad):
            call()
    qc, e, m = randn(g, 2, 3, 4, 64, dtype=BF), randn(g, 2, 20, 2, 64, dtype=BF), torch.ones(2, 3, 4, dtype=torch.uint8, device="cuda")
    for call in [lambda: tq.tq_cross_attention(qc, e, e[:, :19], ws), lambda: tq.tq_cross_attention(qc, e[:1], e[:1], ws),
                 lambda: tq.tq_cross_attention(qc, e, e, ws, mask=m, block_len=4), lambda: tq.tq_cross_attention(qc, e, e, ws, mask=m.int(), block_len=5),
                 lambda: tq.tq_cross_attention(qc[:, :, :3], e, e, ws), lambda: tq.tq_cross_attention(qc, e, e, ws, kv_len=m[0, 0]),
                 lambda: tq.tq_cross_attention(qc, e, e, ws, out=qc[:1])]:
        with pytest.raises(bad):
            call()
