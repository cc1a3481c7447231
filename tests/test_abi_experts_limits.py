"""The expert layer's sizes near its limits, on the host (CPU only)."""
from __future__ import annotations

import ctypes

import pytest

from paper_2110_15456_amd import _lib

LIMIT = (1 << 31) - (1 << 20)


def plan_ws(slots, experts):
    places, ws = ctypes.c_int64(-1), ctypes.c_size_t(0)
    assert _lib.load().bfp_expert_plan_sizes(slots, 1, experts, ctypes.byref(places), ctypes.byref(ws)) == 0
    return ws.value


@pytest.mark.parametrize("experts", [1, 8, 512])
def test_plan_workgroups_are_bounded(experts):
    """Every workgroup of the plan reads the counts of all of them, so that their
    number must not grow with the slots: the workspace holds at most 256 counts of
    each expert and of the dropped slots."""
    most = 256 * (experts + 1) * 4
    for slots in (1 << 20, (1 << 20) + 1, 3 << 19, 1 << 23, 1 << 30, LIMIT - 1, LIMIT):
        ws = plan_ws(slots, experts)
        assert ws % ((experts + 1) * 4) == 0 and most / 2 < ws <= most, (slots, ws)
    # below, one workgroup for each 4096 slots
    for slots in (4097, 8192, 8193, 100000):
        assert plan_ws(slots, experts) == -(-slots // 4096) * (experts + 1) * 4
