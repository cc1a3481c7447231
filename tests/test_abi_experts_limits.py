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


def test_route_arguments():
    lib = _lib.load()
    rows, waves = ctypes.c_int(-9), ctypes.c_int(-9)

    def route(am=4, bm=4, experts=8, slots=64, N=256, K=256, ma=4, mb=4, r=ctypes.byref(rows), w=ctypes.byref(waves)):
        return lib.bfp_gemm_experts_route(am, bm, experts, slots, N, K, ma, mb, r, w)

    def grad(am=4, bm=4, experts=8, M=64, N=256, places=1024, ma=4, mb=4, r=ctypes.byref(rows)):
        return lib.bfp_gemm_experts_grad_route(am, bm, experts, M, N, places, ma, mb, r)

    assert route() == 0 and rows.value in (0, 16, 32, 128) and (waves.value > 0) == (rows.value in (16, 32))
    assert grad() == 0 and rows.value in (0, 128)
    for bad in (dict(r=None), dict(w=None), dict(slots=0), dict(N=0), dict(slots=-1), dict(experts=0)):
        assert route(**bad) == 1, bad
    for bad in (dict(r=None), dict(M=0), dict(N=0), dict(experts=0)):
        assert grad(**bad) == 1, bad
    assert route(K=40) == 2 and grad(places=192) == 2
    assert route(ma=3) == 3 and route(experts=513) == 3 and grad(ma=3) == 3
    assert route(am=9) == 4 and grad(mb=5) == 4


def test_update_route_arguments():
    lib = _lib.load()
    tiles, stages, parts, whole = (ctypes.c_int * 3)(), (ctypes.c_int * 3)(), (ctypes.c_int * 2)(), (ctypes.c_int64 * 2)()
    out = [tiles, stages, parts, whole]
    assert lib.bfp_orthogonalize_route(2, 300, 500, *out) == 0
    assert all(t in (64, 128, 256) for t in tiles) and all(s in (2, 4) for s in stages) and min(parts) >= 1
    turned = [type(o)() for o in out]
    assert lib.bfp_orthogonalize_route(2, 500, 300, *turned) == 0 and list(map(list, out)) == list(map(list, turned))
    for i in range(4):
        assert lib.bfp_orthogonalize_route(2, 300, 500, *[None if j == i else o for j, o in enumerate(out)]) == 1
    assert lib.bfp_orthogonalize_route(0, 300, 500, *out) == 1 and lib.bfp_orthogonalize_route(1, 0, 5, *out) == 1
    assert lib.bfp_orthogonalize_route(1, 1 << 20, 16, *out) == 3
