"""The expert layer's calls at the edges of what they take."""
from __future__ import annotations

import pytest
import torch

import paper_2110_15456_amd as fb
from gpu_util import announce

pytestmark = pytest.mark.gpu


def test_weighted_sum_over_its_input():
    """One choice a token: out has y's shape, but the rows change places."""
    announce("weighted sum over its input is refused")
    p = fb.expert_plan(torch.tensor([2, 0, 1, 0], device="cuda"), 3)
    y = torch.randn((4, 32), device="cuda")
    with pytest.raises(fb.BFPError):
        fb.combine_experts(y, p, out=y)
    with pytest.raises(fb.BFPError):
        fb.combine_experts_grad(y, y.clone(), p, out=y)
