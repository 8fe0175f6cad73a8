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
