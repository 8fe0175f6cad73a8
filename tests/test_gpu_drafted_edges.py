"""The operators of a decode step with drafted tokens where their inputs are unusual.  References, helpers and what is not said here of
bounds are those of test_gpu_drafted.py."""
import pytest
import torch

from test_gpu_drafted import f32, gen, i32, logits, randn, sample_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tq():
    from paper_2509_22951_b200 import binding
    return binding


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
