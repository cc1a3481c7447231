"""The expert layer's calls at the edges of what they take."""
from __future__ import annotations

import numpy as np
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


# Beyond 2^20 slots a workgroup of the plan takes several rounds.
@pytest.mark.parametrize("slots,experts,dtype", [(1 << 20, 8, torch.int32), ((1 << 20) + 1, 8, torch.int64),
                                                 (2500001, 130, torch.int32), (4194305, 512, torch.int64)])
def test_plan_of_many_slots(slots, experts, dtype):
    announce("plan of %d slots, %d experts" % (slots, experts))
    rng = np.random.Generator(np.random.PCG64(slots))
    ids = np.minimum(rng.geometric(2.0 / experts, slots) - 1, experts)  # skewed; the id past the end: dropped
    p = fb.expert_plan(torch.from_numpy(ids).to(dtype).cuda(), experts)
    counts = np.bincount(ids, minlength=experts + 1)[:experts]
    order = np.argsort(ids, kind="stable")
    assert np.array_equal(p.offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(counts)]))
    assert np.array_equal(p.k_offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(-(-counts // 128) * 128)]))
    assert np.array_equal(p.order.cpu().numpy(), order)
    place = np.empty_like(order)
    place[order] = np.arange(slots)
    assert np.array_equal(p.place.cpu().numpy(), place)
