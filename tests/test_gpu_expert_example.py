"""The example's expert layer learns: its loss falls by half within 40 steps at 4 and
6 bits (it starts at the power of the target plus that of an untrained layer)."""
from __future__ import annotations

import math
import os
import sys

import pytest

from gpu_util import announce

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("m", [4, 6])
def test_example_learns(m):
    import expert_ffn
    announce("example expert layer at %d bits" % m)
    losses = expert_ffn.train(steps=40, tokens=1024, m=m, log=lambda s: print(s, flush=True))
    assert all(math.isfinite(v) for v in losses)
    assert losses[-1] < 0.5 * losses[0], losses
