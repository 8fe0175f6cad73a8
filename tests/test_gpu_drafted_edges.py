"""The operators of a decode step with drafted tokens where their inputs are unusual.  References, helpers and what is not said here of
bounds are those of test_gpu_drafted.py."""
import math

import pytest
import torch

from test_gpu_drafted import BF, attend_ref, f32, gen, i32, logits, randn, sample_case, within

pytestmark = pytest.mark.gpu
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


# ------------------------------------------------------------------------------------------------ sampling
@pytest.mark.parametrize("mask", [-65504.0, -1e5, -5e4, -3e5])
@pytest.mark.parametrize("lift", [0.0, 30000.0])  # with it the row's largest logit over the temperature leaves the weights' short form
def test_logits_masked_by_a_large_number(tq, mask, lift):
    """Most of a vocabulary masked by a number instead of -inf: t = (x - max) log2(e) / temperature lies between -8e5 and -2e5 for most of these."""
    g, R = gen(int(-mask)), 9
    for vocab in (1000, 50257):
        x, u = logits(g, R, vocab), torch.rand(R, generator=g, device="cuda")
        masked = torch.rand(R, vocab, generator=g, device="cuda") < 0.9
        masked[0] = True
        masked[0, 7] = masked[0, 400] = False
        x = torch.where(masked, mask, x) + lift
        t = f32([0.1, 0.15, 0.2, 0.25, 0.3, 0.1, 0.2, 0.3, 1.0])
        sample_case(tq, x, u, temperature=t)
        sample_case(tq, x, u, temperature=t, top_p=f32([0.3, 0.9, 0.999] * 3))
        sample_case(tq, x, u, temperature=t, top_k=i32([50, 1, 300, 1000, 20, 2, 700, 100, 5]))
        sample_case(tq, x, u, temperature=t, top_k=i32([1100, 2000, 5000] * 3))
        sample_case(tq, x, u, temperature=t, min_p=f32([0.01, 0.3, 1e-30] * 3))


def test_top_k_of_logits_next_to_one_another(tq):
    """Logits whose distances are subnormal numbers, or so unlike that a bin's width over the first hundreds is nothing against the rest."""
    g, V = gen(71), 20000
    x = torch.zeros(6, V, device="cuda")
    x[0] = 1e-41 * torch.arange(V, device="cuda")
    x[1] = -1e-41 * torch.arange(V, device="cuda")
    x[2, 1234] = 1e-38
    x[3, 77:] = -1e-39
    x[4, ::3] = 1e-45
    x[5] = torch.randn(V, generator=g, device="cuda") * 1e-37
    u = torch.rand(6, generator=g, device="cuda")
    for k in (1, 2, 50, 1000):
        for t in (1e-36, 1.0, 1e30):
            for v in (u, torch.full_like(u, 1.0 - 2.0 ** -24)):
                sample_case(tq, x, v, top_k=i32([k] * 6), temperature=f32([t] * 6))
                sample_case(tq, x, v, top_k=i32([k] * 6), temperature=f32([t] * 6), top_p=f32([0.6] * 6), min_p=f32([0.1] * 6))
    # a thread's largest logits next to one another, its others far below, and as likely at this temperature: fewer of the first than k
    for V in (600, 1200):
        y = torch.full((4, V), -1e9, device="cuda")
        y[:, ::4] = torch.where(torch.arange(V // 4, device="cuda") % 2 == 0, 0.0, -1e-30)
        v = f32([0.1, 0.5, 0.9, 1.0 - 2.0 ** -24])
        sample_case(tq, y, v, top_k=i32([V // 4 + 50] * 4), temperature=f32([1e30] * 4))
        sample_case(tq, y, v, top_k=i32([V - 1] * 4), temperature=f32([1e30] * 4))


# ------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("D,H,n", [(64, 4, 5), (128, 4, 5), (64, 16, 40), (128, 16, 40)])  # tiles of 128 rows and of 256
@pytest.mark.parametrize("page", [16, 20])  # tensor copies, copies row by row
def test_pages_outside_the_pool_are_zeros(tq, ws, D, H, n, page):
    """What is multiplied with p = 0 in their place does not come from what the multiprocessor had before: the same bits after values of all kinds."""
    g, K = gen(D + n + page), 2
    P = 320 // page
    kp, vp = randn(g, P, K, page, D, dtype=BF), randn(g, P, K, page, D, dtype=BF)
    cache, q = tq.tq_kv_cache(kp, vp), randn(g, n, H, D, dtype=BF)
    table = torch.arange(P, device="cuda", dtype=torch.int32)[None].contiguous()
    table[0, [1, 7, 9]] = i32([-1, P, 2 ** 31 - 1])
    args = (q, cache, table, i32([0, n]), i32([300]), ws)
    # every stage of every multiprocessor
    B = 400
    dirty = [tq.tq_kv_cache(torch.zeros_like(kp), torch.full_like(vp, v)) for v in (0.0, INF, NAN)]
    many = torch.arange(P, device="cuda", dtype=torch.int32).expand(B, -1).contiguous()
    got = []
    for d in dirty:
        tq.tq_tree_attention(torch.zeros(B * n, H, D, dtype=BF, device="cuda"), d, many, i32([n * b for b in range(B + 1)]), i32([320] * B), ws)
        got.append(tq.tq_tree_attention(*args))
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    assert tq.tq_kv_cache_status(cache) == tq.TQ_STATUS_BAD_PAGE
    there = torch.ones(P, page, dtype=torch.bool, device="cuda")
    there[[1, 7, 9]] = False
    seen = (there.flatten()[:300] & torch.ones(n, 300, dtype=torch.bool, device="cuda").tril(300 - n))
    for h in range(H):
        k, v = (x[:, h // (H // K)].reshape(-1, D)[:300] for x in (kp, vp))
        want, _, bound = attend_ref(q[:, h], k, v, seen, D ** -0.5)
        within(got[0][:, h], want, bound)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,n", [(4, 7), (16, 9), (16, 40)])  # the last with 256 rows a tile
@pytest.mark.parametrize("length", [1, 70, 900])
def test_an_infinite_value_makes_its_column_infinite(tq, ws, D, H, n, length):
    """Seen by all, with every p above 0: its own column and no other."""
    g, K, page = gen(D + n + length), 2, 16
    P = 60
    kp, vp = randn(g, P, K, page, D, dtype=BF, scale=0.2), randn(g, P, K, page, D, dtype=BF)
    vp[0, :, 0, 5], vp[0, :, 0, 9] = INF, -INF
    kp[0, 0, 0] = kp[0, 0, 0] * 30
    table = torch.arange(P, device="cuda", dtype=torch.int32)[None].contiguous()
    q = randn(g, n, H, D, dtype=BF)
    out = tq.tq_tree_attention(q, tq.tq_kv_cache(kp, vp), table, i32([0, n]), i32([length + n - 1]), ws)
    assert bool((out[..., 5] == INF).all()) and bool((out[..., 9] == -INF).all())
    others = [c for c in range(D) if c not in (5, 9)]
    assert bool(out[..., others].isfinite().all())


@pytest.mark.parametrize("D,H,n,length", [(128, 32, 40, 9000), (64, 32, 40, 9000), (128, 8, 3, 20000)])
def test_a_workspace_of_the_stated_size_is_enough(tq, D, H, n, length):
    """Parts of cut groups of both forms: nothing behind the workspace's stated size is written."""
    g, K, page = gen(length), 8, 32
    P = -(-length // page)
    cache = tq.tq_kv_cache(randn(g, P, K, page, D, dtype=BF), randn(g, P, K, page, D, dtype=BF))
    w = tq.tq_attn_workspace()
    room = torch.full((w.bytes + (1 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    room[:w.bytes] = 0
    assert room.data_ptr() % 256 == 0
    w.ptr = room.data_ptr()
    q, table = randn(g, n, H, D, dtype=BF), torch.arange(P, device="cuda", dtype=torch.int32)[None].contiguous()
    out = tq.tq_tree_attention(q, cache, table, i32([0, n]), i32([length]), w)
    assert bool(out.isfinite().all()) and bool((room[w.bytes:] == 0x5A).all())


# ------------------------------------------------------------------------------------------------ the binding
def test_settings_of_any_shape(tq, monkeypatch):
    """A setting is `rows` numbers one behind the other, in whatever shape, for both forms of a call."""
    g, R, V = gen(72), 6, 3000
    x, u = randn(g, R, V, scale=3), torch.rand(R, generator=g, device="cuda")
    kw = dict(temperature=f32([0.7] * R), top_k=i32([40] * R), top_p=f32([0.9] * R), min_p=f32([0.01] * R))
    first, lens, tokens, parents, sampled = i32([0, 4, 6]), i32([40, 20]), i32([1, 2, 3, 4, 5, 6]), i32([-1, 0, 1, 0, -1, 0]), i32([2, 3, 4, 4, 6, 6])
    want, path = tq.tq_sample(x, u, **kw), tq.tq_tree_accept(None, None, first, lens, tokens, parents, sampled, 3)
    for form in (tq._fast, None):
        monkeypatch.setattr(tq, "_fast", form)
        for shape in ((R, 1), (1, R), (2, 3)):
            other = {n: v.view(shape) for n, v in kw.items()}
            assert torch.equal(tq.tq_sample(x, u, **other), want)
            assert torch.equal(tq.tq_sample(x, u, out=torch.empty_like(want), **other), want)
            assert torch.equal(tq.tq_sample(x, u, logprob=torch.empty(R, device="cuda"), **other)[0], want)
        got = tq.tq_tree_accept(None, None, first, lens, tokens, parents.view(6, 1), sampled.view(2, 3), 3)
        assert all(torch.equal(a, b) for a, b in zip(got, path))
        for bad in (u[:5], x[0, :12].view(6, 2), u.view(R, 1).expand(R, 2)):
            with pytest.raises(AssertionError):
                tq.tq_sample(x, u, temperature=bad)
