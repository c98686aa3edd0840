"""Scalings that a rotation plan cannot mean are refused (no GPU needed)."""
import pytest
import torch

from paper_2607_17644_b200 import laga


@pytest.mark.parametrize("scaling", [{"factor": 40}, {"type": "yarn"}, {"type": "linear"}, {"type": "ntk", "original_length": 4096},
                                     {"type": "none", "factor": 8}, {"type": "yarn", "factor": float("nan")},
                                     {"type": "yarn", "factor": float("inf")}, {"type": "yarn", "factor": 2, "original_length": 0}])
def test_scalings_that_are_refused(scaling):
    with pytest.raises(ValueError):
        laga.rope_plan(64, scaling=scaling, device="cpu")


def test_scalings_that_are_not():
    plain = laga.rope_plan(64, device="cpu")
    for scaling in ({"type": "none"}, {"type": "none", "factor": 1}, {"type": "linear", "factor": 1}, {"type": "ntk", "factor": 1},
                    {"type": "yarn", "factor": 1}):
        plan = laga.rope_plan(64, scaling=scaling, device="cpu")
        assert torch.allclose(plan.freqs, plain.freqs, rtol=1e-15) and plan.mscale == 1.0
