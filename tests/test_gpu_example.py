"""The decoder of examples/vision_decoder.py: compressed products and the operators between them, against the formulas in
64 bits."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "vision_decoder.py")


@pytest.mark.parametrize("batch,steps,layers", [(1, 20, "scs"), (3, 40, "sc"), (5, 17, "s")])
def test_decoder_follows_the_formulas(batch, steps, layers):
    import sys

    spec = importlib.util.spec_from_file_location("vision_decoder", PATH)
    ex = importlib.util.module_from_spec(spec)
    sys.modules["vision_decoder"] = ex  # dataclasses look their module up
    spec.loader.exec_module(ex)
    tokens, error, _ = ex.run(ex.Config(layers=layers), batch, steps)
    assert tokens.shape == (batch, steps) and int(tokens.max()) < 1024
    # about a dozen roundings to bf16 (2^-8 at most, 2^-9.8 rms, of independent elements) lie between the embedding and the logits
    # of each layer; a logit is a sum of 256 such products, and the largest of 1024 errors is some 4 of their deviations:
    # 4 * sqrt(12 * layers) * 2^-9.8 of a logit's own deviation, a third of the largest logit
    assert error <= 4 * (12 * len(layers)) ** 0.5 * 2.0 ** -9.8 / 3 * 2, error
