"""Arguments that nobody holds but the call: their memory must not become the result's before the call has used them.  A freed block is
the first that an allocation of the same size class gets, so a result would lie in the arguments: the addresses that reach the library
are compared."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


class Spy:
    """The library, with the arguments of its last call."""

    def __init__(self, lib):
        self._spied, self.args = lib, None

    def __getattr__(self, name):
        fn = getattr(self._spied, name)

        def call(*args):
            self.args = args
            return fn(*args)
        return call


@pytest.fixture
def tq(monkeypatch):
    from paper_2509_22951_b200 import binding
    monkeypatch.setattr(binding, "_fast", None)  # the native form holds its arguments
    monkeypatch.setattr(binding, "_lib", Spy(binding._lib))
    yield binding
    torch.cuda.synchronize()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def apart(args, results):
    """No address of a result among the other arguments; every result here is a block of 512 bytes of its own."""
    torch.cuda.synchronize()
    at = [a for a in args if isinstance(a, int) and a > 1 << 32]
    for r in results:
        assert at.count(r.data_ptr()) == 1
    return True


def rand(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def test_cross_attention(tq):
    g = torch.Generator(device="cuda").manual_seed(1)
    ws, k = tq.tq_attn_workspace(), rand(g, 4, 30, 1, 64, dtype=BF)
    out = tq.tq_cross_attention(rand(g, 4, 1, 1, 64, dtype=BF), k, k.clone(), ws, kv_len=i32([30, 20, 10, 7]), mask=torch.ones(4, 1, 3, dtype=torch.uint8, device="cuda"),
                                block_len=10)
    assert apart(tq._lib.args, [out])


def test_the_sum_of_a_norm(tq):
    g = torch.Generator(device="cuda").manual_seed(2)
    h, d, w = rand(g, 2, 128, dtype=BF), rand(g, 2, 128), torch.ones(128, device="cuda")
    assert apart((out := tq.tq_rmsnorm(h, w, d, h_out=torch.empty_like(h)), tq._lib.args)[1], [out])
    q, s = tq.tq_rmsnorm_q8(h, w, d, h_out=torch.empty_like(h))
    assert apart(tq._lib.args, [q, s])


def test_tree_attention(tq):
    g = torch.Generator(device="cuda").manual_seed(3)
    cache, ws = tq.tq_kv_cache(rand(g, 8, 1, 16, 64, dtype=BF), rand(g, 8, 1, 16, 64, dtype=BF)), tq.tq_attn_workspace()
    q = rand(g, 4, 1, 64, dtype=BF)
    want = tq.tq_tree_attention(q, cache, table := i32([[0, 1, 2], [5, 6, 7]]), first := i32([0, 2, 4]), lens := i32([40, 20]), ws, mask=(mask := i32([[1], [3], [1], [3]])))
    out = tq.tq_tree_attention(q, cache, table.clone(), first.clone(), lens.clone(), ws, mask=mask.clone())
    assert apart(tq._lib.args, [out]) and torch.equal(out, want)


def test_sample_and_accept(tq):
    g = torch.Generator(device="cuda").manual_seed(4)
    x, p = rand(g, 4, 1000), lambda: torch.full((4,), 0.9, device="cuda")  # noqa: E731
    out = tq.tq_sample(x, p(), temperature=p(), top_k=i32([5] * 4), top_p=p(), min_p=p(), logprob=True)
    assert apart(tq._lib.args, out)
    out = tq.tq_tree_accept(None, None, i32([0, 2, 4]), i32([40, 20]), i32([1, 2, 3, 4]), i32([-1, 0, -1, 0]), i32([2, 2, 4, 4]), 4)
    assert apart(tq._lib.args, out) and out[2].tolist() == [2, 2]


def test_heads(tq):
    g = torch.Generator(device="cuda").manual_seed(5)
    cache = tq.tq_kv_cache(rand(g, 8, 1, 16, 64, dtype=BF), rand(g, 8, 1, 16, 64, dtype=BF))
    one = lambda: torch.ones(64, device="cuda")  # noqa: E731
    out = tq.tq_qk_norm_rope_append(rand(g, 2, 1, 64), rand(g, 2, 1, 64), rand(g, 2, 1, 64), one(), one(), rand(g, 2, 64), i32([0, 1]), i32([0, 1]), cache)
    assert apart(tq._lib.args, [out])
    out = tq.tq_rope_append(rand(g, 2, 1, 64), rand(g, 2, 1, 64), rand(g, 2, 1, 64), rand(g, 2, 64), i32([0, 1]), i32([0, 1]), cache)
    assert apart(tq._lib.args, [out])
