"""Limits of examples/vision_decoder.py, decided on the host before anything is launched."""
import importlib.util
import os
import sys

import pytest
import torch

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "vision_decoder.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("vision_decoder", PATH)
    m = importlib.util.module_from_spec(spec)
    sys.modules["vision_decoder"] = m  # dataclasses look their module up
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("steps", [0, -1, 257])
def test_run_takes_as_many_steps_as_the_cache_holds(ex, steps, monkeypatch):
    def made(*a):
        raise AssertionError("nothing is to be made")

    monkeypatch.setattr(ex, "Decoder", made)
    with pytest.raises(ValueError):
        ex.run(ex.Config(max_tokens=256), 1, steps)


def test_a_step_past_the_page_table_is_refused(ex):
    """On a decoder whose sequences are full, all of its tensors on the CPU: the refusal comes before the first operation."""
    d = ex.Decoder.__new__(ex.Decoder)
    d.cfg, d.batch, d.steps = ex.Config(), 2, ex.Config().max_tokens
    d.lens = torch.full((2,), d.steps, dtype=torch.int32)
    with pytest.raises(ValueError):
        d.step(torch.zeros(2, dtype=torch.int64))
    assert d.steps == d.cfg.max_tokens and d.lens.tolist() == [d.steps] * 2
