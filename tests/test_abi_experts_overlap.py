"""Outputs of the expert layer that share memory with what their kernels read are
rejected on the host, before any launch.  CPU only: a call that is accepted here
would reach the HIP runtime, so every call below is one that must be refused."""
from __future__ import annotations

import ctypes

import pytest

from paper_2110_15456_amd import _lib

E_ARG = 1
TOKENS, TOP, EXPERTS, N = 8, 2, 4, 16
SLOTS = TOKENS * TOP
# base and bytes of each array, far apart
AT = dict(y=(0x1000000, SLOTS * N * 4), gates=(0x2000000, SLOTS * 4), place=(0x3000000, SLOTS * 4),
          offsets=(0x4000000, (EXPERTS + 1) * 4), dout=(0x5000000, TOKENS * N * 4), out=(0x6000000, TOKENS * N * 4),
          dy=(0x7000000, SLOTS * N * 4), dgates=(0x8000000, SLOTS * 4))


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def ends(written, read):
    """Places of `written` that share its first, its last or all of its bytes with `read`."""
    size, (base, n) = AT[written][1], AT[read]
    return [base, base + n - 4, base - size + 4]


@pytest.mark.parametrize("read", ["y", "gates", "place", "offsets"])
def test_weighted_sum(lib, read):
    for at in ends("out", read):
        p = {k: ctypes.c_void_p(v[0]) for k, v in AT.items()}
        assert lib.bfp_combine_experts(p["y"], p["gates"], p["place"], p["offsets"], TOKENS, TOP, EXPERTS, N,
                                       ctypes.c_void_p(at), None) == E_ARG, hex(at)


def test_weighted_sum_in_place(lib):
    """One choice a token: out has y's shape, and in place would be a permutation."""
    y, place, offsets = (ctypes.c_void_p(AT[k][0]) for k in ("y", "place", "offsets"))
    assert lib.bfp_combine_experts(y, None, place, offsets, SLOTS, 1, EXPERTS, N, y, None) == E_ARG


@pytest.mark.parametrize("written", ["dy", "dgates"])
@pytest.mark.parametrize("read", ["y", "gates", "place", "offsets", "dout", "other"])
def test_gradients(lib, written, read):
    other = "dgates" if written == "dy" else "dy"
    for at in ends(written, other if read == "other" else read):
        p = {k: ctypes.c_void_p(v[0]) for k, v in AT.items()}
        p[written] = ctypes.c_void_p(at)
        assert lib.bfp_combine_experts_grad(p["dout"], p["y"], p["gates"], p["place"], p["offsets"], TOKENS, TOP,
                                            EXPERTS, N, p["dy"], p["dgates"], None) == E_ARG, hex(at)


@pytest.mark.parametrize("over", ["grad", "momentum", "momentum_out", "out"])
def test_workspace_of_the_update(lib, over):
    """The update's workspace is overwritten: not over what it reads or writes."""
    batch, rows, cols = 2, 64, 128
    need = ctypes.c_size_t(0)
    assert lib.bfp_orthogonalize_ws_size(batch, rows, cols, ctypes.byref(need)) == 0
    size = batch * rows * cols * 4  # (a multiple of 256, as the workspace's places are)
    at = dict(grad=0x10000000, momentum=0x20000000, momentum_out=0x30000000, out=0x40000000)
    p = {k: ctypes.c_void_p(v) for k, v in at.items()}
    assert need.value % 256 == 0
    for ws in (at[over], at[over] + size - 256, at[over] - need.value + 256):
        assert lib.bfp_orthogonalize(p["grad"], p["momentum"], p["momentum_out"], 0.9, 1, batch, rows, cols, 5, 1e-7,
                                     p["out"], ctypes.c_void_p(ws), need, None) == E_ARG, hex(ws)
