"""The expert layer's and the orthogonalised update's entry points: sizes, and bad
arguments rejected on the host before any launch.  CPU only: every call here
returns before touching the HIP runtime."""
from __future__ import annotations

import ctypes
import itertools

import pytest

from paper_2110_15456_amd import _lib

OK, E_ARG, E_SHAPE, E_UNSUP, E_PREC, E_HIP = range(6)
FAKE = ctypes.c_void_p(0x100000)  # never dereferenced
ODD = ctypes.c_void_p(0x100002)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def sizes(lib, tokens, top, experts):
    places, ws = ctypes.c_int64(-1), ctypes.c_size_t(99)
    st = lib.bfp_expert_plan_sizes(tokens, top, experts, ctypes.byref(places), ctypes.byref(ws))
    return st, places.value, ws.value


def test_plan_sizes(lib):
    assert sizes(lib, 0, 2, 8) == (OK, 0, 0)
    assert sizes(lib, 1, 1, 1) == (OK, 128, 0)
    # every way of sharing few slots over few experts fits, and the worst one exactly
    for slots, experts in ((1, 3), (2, 2), (5, 3), (130, 2), (257, 3)):
        worst = 0
        for cut in itertools.product(range(slots + 1), repeat=experts):
            if sum(cut) <= slots:
                worst = max(worst, sum(-(-n // 128) * 128 for n in cut))
            if experts > 2 and slots > 200 and cut[0] > 3:
                break
        st, places, _ = sizes(lib, slots, 1, experts)
        assert st == OK and places % 128 == 0 and places >= worst
        if slots <= 130:
            assert places == worst
    assert sizes(lib, 4096, 1, 8)[2] == 0 and sizes(lib, 4097, 1, 8)[2] == 2 * 9 * 4  # (a second workgroup's counts)
    assert sizes(lib, 4, 2, 512)[0] == OK and sizes(lib, 4, 2, 513)[0] == E_UNSUP
    assert sizes(lib, 4, 2, 0)[0] == E_ARG and sizes(lib, 4, 0, 8)[0] == E_ARG and sizes(lib, -1, 2, 8)[0] == E_ARG
    assert sizes(lib, 1 << 30, 2, 8)[0] == E_UNSUP
    assert lib.bfp_expert_plan_sizes(4, 2, 8, None, None) == E_ARG


def plan(lib, ids=FAKE, bits=64, tokens=4, top=2, experts=8, off=FAKE, koff=FAKE, order=FAKE, place=FAKE, ws=None, n=0):
    return lib.bfp_expert_plan(ids, bits, tokens, top, experts, off, koff, order, place, ws, n, None)


def test_plan_refusals(lib):
    for bad in (dict(ids=None), dict(off=None), dict(koff=None), dict(order=None), dict(place=None), dict(bits=16),
                dict(ids=ctypes.c_void_p(0x100004)), dict(order=ODD), dict(tokens=5000, ws=None, n=1 << 20),
                dict(tokens=5000, ws=FAKE, n=8), dict(experts=0)):
        assert plan(lib, **bad) == E_ARG, bad
    assert plan(lib, experts=513) == E_UNSUP


def quant(lib, x=FAKE, C=64, gather=1, order=FAKE, off=FAKE, koff=FAKE, tokens=4, top=2, experts=8, m=4, mode=0,
          mr=FAKE, er=FAKE, mc=FAKE, ec=FAKE, st=None):
    return lib.bfp_quantize_experts(x, C, gather, order, off, koff, tokens, top, experts, m, mode, 0, 0, mr, er, mc, ec,
                                    st, None)


def test_quantize_refusals(lib):
    for bad in (dict(x=None), dict(order=None), dict(off=None), dict(koff=None), dict(gather=2), dict(mode=3),
                dict(er=None), dict(mc=None), dict(mr=None, er=None, mc=None, ec=None), dict(x=ODD), dict(mr=ODD),
                dict(x=ctypes.c_void_p(0x100004)), dict(tokens=-1), dict(C=-16)):
        assert quant(lib, **bad) == E_ARG, bad
    assert quant(lib, C=40) == E_SHAPE
    assert quant(lib, m=0) == E_PREC and quant(lib, m=9) == E_PREC
    assert quant(lib, C=1 << 22) == E_UNSUP
    assert quant(lib, tokens=1 << 20, top=64, C=1024) == E_UNSUP  # 2^31 groups and more
    assert quant(lib, tokens=0) == OK and quant(lib, C=0) == OK


def gemm(lib, a=FAKE, ae=FAKE, am=4, b=FAKE, be=FAKE, bm=4, off=FAKE, experts=8, slots=4, N=8, K=64, ma=4, mb=4,
         C=FAKE, ldc=8):
    return lib.bfp_gemm_experts(a, ae, am, b, be, bm, off, experts, slots, N, K, ma, mb, C, ldc, None)


def test_gemm_refusals(lib):
    for bad in (dict(a=None), dict(b=None), dict(ae=None), dict(be=None), dict(off=None), dict(C=None), dict(a=ODD),
                dict(C=ODD), dict(off=ODD), dict(slots=-1), dict(N=-1), dict(K=-16), dict(experts=0)):
        assert gemm(lib, **bad) == E_ARG, bad
    assert gemm(lib, K=40) == E_SHAPE and gemm(lib, ldc=7) == E_SHAPE
    assert gemm(lib, am=9) == E_PREC and gemm(lib, ma=5) == E_PREC and gemm(lib, mb=0) == E_PREC
    assert gemm(lib, ma=3) == E_UNSUP and gemm(lib, bm=8, mb=5) == E_UNSUP  # between chunk boundaries
    assert gemm(lib, experts=513) == E_UNSUP
    kmax = ((1 << 31) // (256 * 12) - 1) * 16
    assert gemm(lib, K=kmax + 16) == E_UNSUP
    assert gemm(lib, slots=(1 << 30), N=(1 << 31) - 1, ldc=(1 << 31) - 1) == E_UNSUP
    assert gemm(lib, slots=0) == OK and gemm(lib, N=0, ldc=0) == OK
    assert gemm(lib, slots=0, am=8, ma=4, bm=6, mb=4) == OK  # low chunks dropped


def grad(lib, a=FAKE, ae=FAKE, am=4, b=FAKE, be=FAKE, bm=4, koff=FAKE, experts=8, M=16, N=16, places=256, ma=4, mb=4,
         C=FAKE):
    return lib.bfp_gemm_experts_grad(a, ae, am, b, be, bm, koff, experts, M, N, places, ma, mb, C, None)


def test_grad_refusals(lib):
    for bad in (dict(a=None), dict(b=None), dict(ae=None), dict(be=None), dict(koff=None), dict(C=None), dict(ae=ODD),
                dict(be=ODD), dict(M=-1), dict(places=-128)):
        assert grad(lib, **bad) == E_ARG, bad
    assert grad(lib, places=192) == E_SHAPE
    assert grad(lib, ma=3) == E_UNSUP and grad(lib, experts=600) == E_UNSUP
    assert grad(lib, M=1 << 24, N=1 << 22) == E_UNSUP  # more workgroups than a grid holds
    assert grad(lib, am=0) == E_PREC
    assert grad(lib, M=0) == OK


def test_combine_refusals(lib):
    def fwd(y=FAKE, g=FAKE, place=FAKE, off=FAKE, tokens=4, top=2, experts=8, N=16, out=FAKE):
        return lib.bfp_combine_experts(y, g, place, off, tokens, top, experts, N, out, None)

    def bwd(dout=FAKE, y=ctypes.c_void_p(0x200000), g=FAKE, place=FAKE, off=FAKE, tokens=4, top=2, experts=8, N=16,
            dy=ctypes.c_void_p(0x300000), dg=FAKE):
        return lib.bfp_combine_experts_grad(dout, y, g, place, off, tokens, top, experts, N, dy, dg, None)

    for bad in (dict(y=None), dict(place=None), dict(off=None), dict(out=None), dict(y=ODD), dict(g=ODD), dict(N=-1),
                dict(top=0), dict(tokens=-1)):
        assert fwd(**bad) == E_ARG, bad
    assert fwd(experts=1000) == E_UNSUP and fwd(N=(1 << 31) + 1) == E_UNSUP
    assert fwd(tokens=0) == OK and fwd(N=0) == OK
    for bad in (dict(dout=None), dict(y=None), dict(dy=None), dict(dg=ODD), dict(dy=ctypes.c_void_p(0x200010)),
                dict(dy=ctypes.c_void_p(0x100040)), dict(place=None)):
        assert bwd(**bad) == E_ARG, bad
    assert bwd(tokens=0) == OK


def ws_size(lib, batch, rows, cols):
    n = ctypes.c_size_t(1)
    return lib.bfp_orthogonalize_ws_size(batch, rows, cols, ctypes.byref(n)), n.value


def test_orthogonalize_refusals(lib):
    assert ws_size(lib, 0, 8, 16) == (OK, 0) and ws_size(lib, 2, 0, 16) == (OK, 0)
    st, need = ws_size(lib, 1, 8, 16)
    assert st == OK and need > 2 * 8 * 128
    assert ws_size(lib, 1, 16, 8) == (OK, need)  # the transpose's
    assert ws_size(lib, -1, 8, 16)[0] == E_ARG and ws_size(lib, 1, 1 << 20, 16)[0] == E_UNSUP
    assert ws_size(lib, 1, 1 << 15, 1 << 15)[0] == E_UNSUP and ws_size(lib, 1 << 27, 8, 16)[0] == E_UNSUP
    assert lib.bfp_orthogonalize_ws_size(1, 8, 16, None) == E_ARG
    big = 8 * 16 * 4

    def ortho(g=0x100000, m=None, mo=None, beta=0.9, nest=1, batch=1, rows=8, cols=16, steps=5, eps=1e-7, out=0x200000,
              ws=0x300000, n=need):
        return lib.bfp_orthogonalize(g, m, mo, beta, nest, batch, rows, cols, steps, eps, out, ws, n, None)

    for bad in (dict(g=None), dict(out=None), dict(ws=None), dict(n=need - 1), dict(ws=0x300010), dict(steps=0),
                dict(steps=17), dict(nest=2), dict(eps=-1.0), dict(eps=float("nan")), dict(g=0x100002),
                dict(out=0x100000), dict(out=0x100000 + big - 4), dict(m=0x400000), dict(m=0x400000, mo=0x200000),
                dict(m=0x400000, mo=0x100010), dict(m=0x400000, mo=0x400010), dict(m=0x200000, mo=0x500000),
                dict(batch=-1), dict(rows=-1)):
        assert ortho(**bad) == E_ARG, bad
    assert ortho(rows=1 << 21) == E_UNSUP
    assert ortho(batch=0) == OK and ortho(rows=0) == OK
