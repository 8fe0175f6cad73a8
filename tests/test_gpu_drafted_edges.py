"""The operators of a decode step with drafted tokens where their inputs are unusual.  References, helpers and what is not said here of
bounds are those of test_gpu_drafted.py."""
import pytest
import torch

from test_gpu_drafted import f32, gen, i32, logits, sample_case

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
