"""The operators between the linear layers at the edges of what they take: tiny values, bad indices, cancelling sums, both
sides of the rules that choose a kernel, graphs and streams.  What is not said here of bounds is as in test_gpu_operators.py."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module")
def tq():
    from paper_2509_22951_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("cols", [64, 256, 512, 516])  # 16 and 32 lanes to a row, a block to a row in units and in single columns
@pytest.mark.parametrize("top", [1.0, 3.8e-37, 3.6e-37, 2e-37, 1e-38, 1e-41, 1e-43, 3e-45])
def test_rmsnorm_q8_of_tiny_rows(tq, cols, top):
    """A quarter of a row is +-2 and the rest 0: the mean square is 1 and eps 0, so the normalised row is h * w exactly, and
    scale and levels follow from it by the rule of tq_quantize_rows, in IEEE arithmetic with subnormal numbers."""
    rng = np.random.default_rng(cols)
    w = (rng.uniform(-0.5, 0.5, cols) * top).astype(np.float32)
    w[3] = top / 2
    h = np.zeros((5, cols), dtype=np.float32)
    for r in range(5):
        at = rng.permutation(cols)[:cols // 4]
        if r != 1:
            at[np.argmax(at == 3) if 3 in at else 0] = 3
        h[r, at] = rng.choice([-2.0, 2.0], cols // 4)
    n = h * w
    amax = np.abs(n).max(1)
    scale = amax / np.float32(127)
    scale = np.where(scale == 0, np.float32(1), scale).astype(np.float32)
    want = np.clip(np.rint(n / scale[:, None]), -127, 127).astype(np.int8)
    q, s = tq.tq_rmsnorm_q8(torch.from_numpy(h).cuda(), torch.from_numpy(w).cuda(), eps=0.0)
    assert np.array_equal(s.cpu().numpy(), scale)
    assert np.array_equal(q.cpu().numpy(), want)


# ------------------------------------------------------------------------------------------------ cross attention
@pytest.fixture(scope="module")
def ws(tq):
    w = tq.tq_attn_workspace()
    yield w
    assert tq.tq_attn_status(w) == 0


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def test_cross_attention_that_gave_up_writes_its_outputs_alone(tq, ws):
    """A call with more groups than entries numbers them by CTA; the call after it has two groups, its entries' places still hold
    the first call's, and its loaders give up before they write theirs."""
    g = gen(1)
    B, T, S, K, D = 9, 20, 1500, 64, 64
    k, v = randn(g, B, S, K, D, dtype=BF), randn(g, B, S, K, D, dtype=BF)
    lens = torch.tensor([1500, 3, 700, 1500, 1100, 0, 900, 1499, 128], dtype=torch.int32, device="cuda")
    tq.tq_cross_attention(randn(g, B, T, K, D, dtype=BF), k, v, ws, kv_len=lens)
    entries = ws.buf[512 * 4 + 256:][:512 * 16].view(torch.int32).view(512, 4)
    assert bool(((entries[:2, 0] > 1) & (entries[:2, 2] >= 2)).any())  # an entry that a block of the next call would find

    q, k, v = randn(g, 1, 17, 2, D, dtype=BF), randn(g, 1, 300, 2, D, dtype=BF), randn(g, 1, 300, 2, D, dtype=BF)
    good = tq.tq_cross_attention(q, k, v, ws)
    tq.tq_cross_attention(randn(g, B, T, K, D, dtype=BF), randn(g, B, S, K, D, dtype=BF), randn(g, B, S, K, D, dtype=BF), ws, kv_len=lens)
    n, room = q.numel(), 1 << 20
    out, lse = torch.full((n + room,), 7.0, dtype=BF, device="cuda"), torch.full((34 + room,), 7.0, device="cuda")
    o, ls = out[:n].view(q.shape), lse[:34].view(1, 17, 2)
    tq.tq_test_withhold_cross_entry(True)
    try:
        tq.tq_cross_attention(q, k, v, ws, out=o, lse=ls)
        torch.cuda.synchronize()
    finally:
        tq.tq_test_withhold_cross_entry(False)
    assert tq.tq_attn_status(ws) == tq.TQ_STATUS_WAIT_EXPIRED
    assert bool((out[n:] == 7.0).all()) and bool((lse[34:] == 7.0).all())
    assert torch.equal(tq.tq_cross_attention(q, k, v, ws, out=o, lse=ls), good)  # the workspace is as good as before
    assert tq.tq_attn_status(ws) == 0


# ------------------------------------------------------------------------------------------------ rotary positions, cache write
@pytest.mark.parametrize("slot,bad", [(-1, False), (-2, True), (-2 ** 31, True), (31, False), (32, True), (2 ** 31 - 1, True)])
def test_rope_append_says_which_slots_are_out_of_range(tq, slot, bad):
    """-1 is padding; every other slot outside the pool sets the bit, alone among good ones."""
    g = gen(2)
    kp, vp = randn(g, 2, 1, 16, 64, dtype=BF), randn(g, 2, 1, 16, 64, dtype=BF)
    k0, v0 = kp.clone(), vp.clone()
    cache = tq.tq_kv_cache(kp, vp)
    q, k, v, table = randn(g, 3, 2, 64), randn(g, 3, 1, 64), randn(g, 3, 1, 64), torch.cat([torch.ones(4, 32), torch.zeros(4, 32)], 1).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = tq.tq_rope_append(q, k, v, table, i32(0, 1, 2), i32(5, slot, 20), cache)
    assert tq.tq_kv_cache_status(cache) == (tq.TQ_STATUS_BAD_PAGE if bad else 0)
    assert torch.equal(out, q.to(BF))  # angles of 0
    k0[0, 0, 5], v0[0, 0, 5], k0[1, 0, 4], v0[1, 0, 4] = k[0, 0], v[0, 0], k[2, 0], v[2, 0]
    if slot == 31:
        k0[1, 0, 15], v0[1, 0, 15] = k[1, 0], v[1, 0]
    assert torch.equal(kp, k0) and torch.equal(vp, v0)


# ------------------------------------------------------------------------------------------------ attention of one token: p
def _cancelling(g, n, K, D):
    """Keys of small scores and values of both signs: weights are alike and the sums of p v nearly cancel, so that an error of p shows."""
    return randn(g, n, K, D, dtype=BF, scale=0.5), torch.where(torch.rand(n, K, D, generator=g, device="cuda") < 0.5, -1.0, 1.0).to(BF)


def _close(got, q, k, v, scale):
    """The scores' sums of |q k| scale stay below 8: their fp32 errors (128 * 2^-24 * 8 at most) move p by 2^-14 of itself, p's two parts keep
    it to 2^-16, and a weight is a quotient of two such sums: 2^-12.9 of sum p |v| in all, taken as 2^-12, and the result's rounding."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    assert float((q.abs() @ k.abs().t()).max()) * scale < 8
    p = torch.softmax(q @ k.t() * scale, -1)
    out = p @ v
    bound = (p @ v.abs()) * 2.0 ** -12 + out.abs() * 2.0 ** -8
    assert bool(((got.to(F64) - out).abs() <= bound).all()), float(((got.to(F64) - out).abs() - bound).max())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [2, 3, 5, 16, 40])
def test_one_token_holds_p_to_more_than_bf16(tq, ws, D, n):
    g = gen(n + D)
    H, K = 16, 2
    k, v = _cancelling(g, n, K, D)
    q = randn(g, 6, H, D, dtype=BF, scale=0.7)
    cross = tq.tq_cross_attention(q[:, None], k.expand(6, -1, -1, -1), v.expand(6, -1, -1, -1), ws)[:, 0]
    kp, vp = (torch.zeros(n, K, 1, D, dtype=BF, device="cuda") for _ in range(2))
    kp[:, :, 0], vp[:, :, 0] = k, v
    table = torch.arange(n, dtype=torch.int32, device="cuda").expand(6, -1).contiguous()
    paged = tq.tq_paged_attention(q, tq.tq_kv_cache(kp, vp), table, torch.full((6,), n, dtype=torch.int32, device="cuda"), ws)
    for out in (cross, paged):
        for h in range(K):
            hs = slice(h * (H // K), (h + 1) * (H // K))
            _close(out[:, hs].reshape(-1, D), q[:, hs].reshape(-1, D), k[:, h], v[:, h], D ** -0.5)


def test_one_token_and_infinite_values(tq, ws):
    """A value of V that is infinite makes its column infinite (both signs: NaN), and no other; so also where p's lower part is 0 or negative."""
    g = gen(3)
    k, v = _cancelling(g, 40, 1, 64)
    v[0, 0, 1], v[7, 0, 2], v[39, 0, 3] = math.inf, -math.inf, math.inf
    v[3, 0, 4], v[5, 0, 4] = math.inf, -math.inf
    q = randn(g, 4, 3, 64, dtype=BF, scale=0.7)
    for n in (1, 40):  # one state: p is 1
        out = tq.tq_cross_attention(q[:, None], k[:n].expand(4, -1, -1, -1), v[:n].expand(4, -1, -1, -1), ws)[:, 0]
        assert bool((out[..., 1] == math.inf).all())
        if n > 1:
            assert bool((out[..., 2] == -math.inf).all()) and bool((out[..., 3] == math.inf).all()) and bool(out[..., 4].isnan().all())
        assert bool(out[..., 5:].isfinite().all()) and bool(out[..., 0].isfinite().all())


# ------------------------------------------------------------------------------------------------ which kernel a call takes
def tensor_core_kernel(ws, call):
    """Whether the call ran on the tcgen05 kernel, which leaves an entry for every group (or CTA) in the workspace."""
    entries = ws.buf[512 * 4 + 256:][:512 * 16]
    entries.zero_()
    call()
    return bool(entries.any())


@pytest.mark.parametrize("B,S,H,K,D,few,many", [(1, 6404, 64, 8, 128, 6, 8), (4, 1601, 64, 8, 128, 2, 6), (4, 1601, 64, 2, 128, 3, 8), (1, 6404, 64, 2, 128, 8, 17),
                                                (1, 20000, 64, 2, 128, 4, 12), (2, 3000, 32, 2, 64, 8, 16), (1, 500, 32, 8, 64, 16, 17)])
def test_the_faster_kernel_for_few_tokens(tq, ws, B, S, H, K, D, few, many):
    """Sizes at which one kernel was measured to be the faster one by 10 % and more; groups of 4 to 32 heads."""
    g = gen(4)
    k, v = randn(g, B, S, K, D, dtype=BF), randn(g, B, S, K, D, dtype=BF)
    for T, want in ((few, False), (many, True)):
        q = randn(g, B, T, H, D, dtype=BF)
        assert tensor_core_kernel(ws, lambda: tq.tq_cross_attention(q, k, v, ws)) == want, T


# ------------------------------------------------------------------------------------------------ both kernels of cross attention
def on(kernel, tq, ws, monkeypatch):
    """Calls of tq_cross_attention from here on have to run on the tensor-core kernel, or on the other one."""
    call = tq.tq_cross_attention

    def checked(*a, **k):
        got = []
        assert tensor_core_kernel(ws, lambda: got.append(call(*a, **k))) == kernel
        return got[0]

    monkeypatch.setattr(tq, "tq_cross_attention", checked)


@pytest.mark.parametrize("T,kernel", [(9, False), (40, True)])
def test_a_broken_query_stays_by_itself(tq, ws, monkeypatch, T, kernel):
    """A NaN in a query makes its own output NaN and leaves the others within their bound, with a mask (where spoiled rows are looked
    for) and without.  (Not bit for bit: when a row's output is rescaled is decided for 32 rows together.)"""
    from test_gpu_operators import attend_ref, within

    on(kernel, tq, ws, monkeypatch)
    g = gen(6)
    S, H, K, D = 1500, 4, 2, 64
    q, k, v = randn(g, 1, T, H, D, dtype=BF), randn(g, 1, S, K, D, dtype=BF), randn(g, 1, S, K, D, dtype=BF)
    q[0, 4, 1, 3] = float("nan")
    q[0, 5, 3] = float("inf")  # scores of both infinities
    mask = torch.ones(1, T, 15, dtype=torch.uint8, device="cuda")
    mask[0, 4:7, 3] = 0
    for m in (None, mask):
        seen = torch.ones(T, S, dtype=torch.bool, device="cuda") if m is None else m[0].bool().repeat_interleave(100, -1)
        out = tq.tq_cross_attention(q, k, v, ws, mask=m, block_len=100)
        assert bool(out[0, 4, 1].isnan().all()) and bool(out[0, 5, 3].isnan().all())
        for h in range(H):
            ok = torch.tensor([t for t in range(T) if (t, h) not in ((4, 1), (5, 3))], device="cuda")
            want, _, bound = attend_ref(q[0, ok, h], k[0, :, h // 2], v[0, :, h // 2], seen[ok], D ** -0.5)
            within(out[0, ok, h], want, bound)
    assert tq.tq_attn_status(ws) == 0


@pytest.mark.parametrize("T,kernel", [(2, False), (17, True)])
@pytest.mark.parametrize("S,block", [(200, 1), (300, 7), (500, 100), (640, 128), (1000, 1000), (1300, 333), (90, 500)])
def test_masks_on_both_kernels(tq, ws, monkeypatch, T, S, block, kernel):
    from test_gpu_operators import cross_case

    if S > 128 or not kernel:  # a single group of one tile leaves no entry to tell by
        on(kernel, tq, ws, monkeypatch)
    cross_case(tq, ws, 2, T, S, 8, 2, 128, kv_len=[S, max(1, S // 2 + 3)], block=block, seed=1)
    cross_case(tq, ws, 2, T, S, 4, 4, 64, block=block, seed=2, mask_rate=0.1, layout=1)


@pytest.mark.parametrize("T,kernel", [(3, False), (17, True)])
def test_lengths_on_both_kernels(tq, ws, monkeypatch, T, kernel):
    from test_gpu_operators import cross_case

    on(kernel, tq, ws, monkeypatch)
    cross_case(tq, ws, 4, T, 300, 8, 4, 64, kv_len=[0, 1, 300, 129], seed=3)
    cross_case(tq, ws, 3, T, 257, 4, 1, 128, kv_len=[-4, 256, 1000], seed=4, spoil=False)


@pytest.mark.parametrize("T,kernel", [(2, False), (20, True)])
def test_a_long_split_on_both_kernels(tq, ws, monkeypatch, T, kernel):
    from test_gpu_operators import cross_case

    on(kernel, tq, ws, monkeypatch)
    cross_case(tq, ws, 1, T, 20000, 8, 1, 128, seed=7)
    cross_case(tq, ws, 1, T, 20000, 8, 1, 64, seed=8, block=2000)


@pytest.mark.parametrize("B,T,S,H,K,D", [(4, 6, 1601, 64, 8, 128), (4, 16, 1601, 64, 2, 128), (3, 16, 4000, 40, 4, 64), (1, 16, 6404, 36, 2, 128)])
def test_few_tokens_on_the_tensor_core_kernel(tq, ws, monkeypatch, B, T, S, H, K, D):
    """2 to 16 tokens over so many states that the tensor-core kernel takes them."""
    from test_gpu_operators import cross_case

    on(True, tq, ws, monkeypatch)
    cross_case(tq, ws, B, T, S, H, K, D, kv_len=[S - 7 * b for b in range(B)], seed=9)
    cross_case(tq, ws, B, T, S, H, K, D, block=401, seed=10)


# ------------------------------------------------------------------------------------------------ graphs and streams
def _calls(tq, g, T):
    """One call of each operator on tensors of its own: -> (run(workspace, cache) writing into `outs`, outs)."""
    h, w, d = randn(g, 5, 512, dtype=BF), randn(g, 512), randn(g, 5, 512)
    q, k, v = randn(g, 5, 4, 64), randn(g, 5, 2, 64), randn(g, 5, 2, 64)
    pos, slots = torch.arange(5, dtype=torch.int32, device="cuda"), torch.tensor([3, 17, -1, 30, 8], dtype=torch.int32, device="cuda")
    pages, lens = torch.tensor([[0, 1]] * 5, dtype=torch.int32, device="cuda"), torch.tensor([20, 9, 0, 32, 1], dtype=torch.int32, device="cuda")
    table = torch.rand(8, 64, generator=g, device="cuda")
    kp, vp = randn(g, 2, 2, 16, 64, dtype=BF), randn(g, 2, 2, 16, 64, dtype=BF)
    cache = tq.tq_kv_cache(kp, vp)
    qc, kc, vc = randn(g, 2, T, 8, 64, dtype=BF), randn(g, 2, 3000, 2, 64, dtype=BF), randn(g, 2, 3000, 2, 64, dtype=BF)
    ho, o, rot = torch.empty_like(h), torch.empty(5, 512, dtype=BF, device="cuda"), torch.empty(5, 4, 64, dtype=BF, device="cuda")
    paged, cross, lse = torch.empty_like(rot), torch.empty_like(qc), torch.empty(2, T, 8, device="cuda")
    outs = [ho, o, rot, kp, vp, paged, cross, lse]

    def run(ws):
        tq.tq_rmsnorm(h, w, d, h_out=ho, out=o)
        tq.tq_rope_append(q, k, v, table, pos, slots, cache, out=rot)
        tq.tq_paged_attention(rot, cache, pages, lens, ws, out=paged)
        tq.tq_cross_attention(qc, kc, vc, ws, out=cross, lse=lse)

    return run, outs


@pytest.mark.parametrize("T", [1, 40])
def test_graphs(tq, ws, T):
    run, outs = _calls(tq, gen(7), T)
    run(ws)
    want = [x.clone() for x in outs]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(ws)
        run(ws)
    for _ in range(3):
        for x in (outs[0], outs[1], outs[2], *outs[5:]):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert tq.tq_attn_status(ws) == 0


@pytest.mark.parametrize("T", [1, 40])
def test_two_streams_with_a_workspace_each(tq, T):
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [tq.tq_attn_workspace(stream=s) for s in streams]
    sets = [_calls(tq, gen(8 + n), T) for n in range(2)]
    want = []
    for (run, outs), space in zip(sets, spaces):
        torch.cuda.synchronize()
        run(space)
        want.append([x.clone() for x in outs])
    for _ in range(5):
        for _, outs in sets:
            for x in (outs[0], outs[1], outs[2], *outs[5:]):
                x.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            for (run, _), space, stream in zip(sets, spaces, streams):
                with torch.cuda.stream(stream):
                    run(space)
        torch.cuda.synchronize()
        for (_, outs), w in zip(sets, want):
            assert all(torch.equal(a, b) for a, b in zip(outs, w))
    assert [tq.tq_attn_status(s) for s in spaces] == [0, 0]


@pytest.mark.parametrize("B,T,S,H,K,D,cut", [(19, 256, 384, 8, 8, 128, True), (10, 256, 640, 16, 16, 128, True), (1, 1024, 6404, 32, 8, 64, True),
                                             (12, 700, 900, 8, 8, 128, False), (3, 1000, 1601, 32, 8, 128, False)])
def test_groups_are_cut_where_that_is_faster(tq, ws, B, T, S, H, K, D, cut):
    """Sizes at which one side was measured to be the faster one (on 148 SMs), and the first and last group's results."""
    from test_gpu_operators import attend_ref, within

    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the shares are those of 148 SMs")
    g = gen(11)
    q, k, v = randn(g, B, T, H, D, dtype=BF), randn(g, B, S, K, D, dtype=BF), randn(g, B, S, K, D, dtype=BF)
    entries = ws.buf[512 * 4 + 256:][:512 * 16].view(torch.int32).view(512, 4)
    entries.zero_()
    out = tq.tq_cross_attention(q, k, v, ws)
    assert bool((entries[:, 0] > 1).any()) == cut
    for b, h in ((0, 0), (B // 2, H // 2), (B - 1, H - 1)):
        want, _, bound = attend_ref(q[b, :, h], k[b, :, h // (H // K)], v[b, :, h // (H // K)], torch.ones(T, S, dtype=torch.bool, device="cuda"), D ** -0.5)
        within(out[b, :, h], want, bound)


@pytest.mark.parametrize("native", [True, False])
def test_one_token_of_a_row_of_any_length(tq, monkeypatch, native):
    """The stride of a single token means nothing, in either form of the call."""
    if not native:
        monkeypatch.setattr(tq, "_fast", None)
    g = gen(12)
    wide = randn(g, 3, 515)
    q, k, v = wide[:1, :256], wide[:1, 256:384], wide[:1, 384:512]
    kp, vp = (torch.zeros(2, 2, 16, 64, dtype=BF, device="cuda") for _ in range(2))
    table = torch.cat([torch.ones(4, 32), torch.zeros(4, 32)], 1).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = tq.tq_rope_append(q, k, v, table, i32(2), i32(17), tq.tq_kv_cache(kp, vp))
    assert torch.equal(out.view(-1), q[0].to(BF)) and torch.equal(kp[1, :, 1].reshape(-1), k[0].to(BF)) and torch.equal(vp[1, :, 1].reshape(-1), v[0].to(BF))
    with pytest.raises(tq.TqError):  # of two tokens it has to be a multiple of 8
        tq.tq_rope_append(wide[:2, :256], wide[:2, 256:384], wide[:2, 384:512], table, i32(1, 2), i32(3, 4), tq.tq_kv_cache(kp, vp))


@pytest.mark.parametrize("cols", [64, 256, 2048, 4096, 8192])
@pytest.mark.parametrize("ht", [BF, F32])
def test_rmsnorm_of_exact_sums_is_that_of_elementary_operations(tq, cols, ht):
    """Small integers in rows of a power of two: the mean square is exact in any order of summation, so scale and levels are those of
    the formula in fp32 operations, bit for bit (the scale by IEEE division, which torch's division by a number is not)."""
    g = gen(13)
    h, w = torch.randint(-8, 9, (300, cols), generator=g, device="cuda").to(ht), randn(g, cols, scale=0.2) + 1
    x = h.float()
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * w
    scale = torch.from_numpy(n.abs().amax(-1).cpu().numpy() / np.float32(127)).cuda()
    q, s = tq.tq_rmsnorm_q8(h, w, eps=1e-5)
    assert torch.equal(s, scale)
    assert torch.equal(q.float(), (n / scale[:, None]).round().clamp(-127, 127))
    assert torch.equal(tq.tq_rmsnorm(h, w, eps=1e-5), n.to(BF))
