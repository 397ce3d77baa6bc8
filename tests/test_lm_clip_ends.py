"""grim_grad_clip where the norm, or the factor that it gives, lies at the ends of fp32 (test_lm_clip.py has the bounds)."""
import math

import pytest
import torch

import paper_2108_11033_amd as g
from test_lm_clip import check, clipped
from lm_helpers import randn


@pytest.mark.gpu
@pytest.mark.parametrize("unscale", [1.0, 0.5])
@pytest.mark.parametrize("place", [False, True])
def test_a_norm_that_fp32_does_not_hold_leaves_gradients_unclipped(unscale, place):
    """Finite gradients whose norm reads as infinity: whoever skips the step by it finds them as they were."""
    grads = [torch.full((9000,), 3e38, device="cuda"), randn(1, 77)]
    before = [t.clone() for t in grads]
    outs = grads if place else [torch.empty_like(t) for t in grads]
    norm, _, _ = clipped(g.GradList(grads, outs), 1.0, unscale)
    assert float(norm) == math.inf
    assert all(torch.equal(a, b * unscale) for a, b in zip(outs, before))
