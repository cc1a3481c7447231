"""What the entry points of the 8-bit blocks, the norm and the clipping refuse, on the
host before any launch.  CPU only."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

import paper_2110_15456_amd as fb
from paper_2110_15456_amd import _lib

OK, E_ARG, E_SHAPE, E_UNSUP, E_PREC, E_HIP = range(6)
P = 1 << 20  # addresses that nothing reads: every call here returns before a launch


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def at(i):
    return P + i * (1 << 24)


def test_sizes(lib):
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    for rows, n, codes, exps in ((3, 1, 384, 12), (2, 128, 256, 8), (2, 129, 512, 8), (1, 513, 640, 8), (0, 5, 0, 0), (4, 0, 0, 0)):
        assert lib.bfp_fp8_sizes(rows, n, ctypes.byref(a), ctypes.byref(b)) == OK
        assert (a.value, b.value) == (codes, exps)
    assert lib.bfp_fp8_sizes(-1, 5, ctypes.byref(a), ctypes.byref(b)) == E_ARG
    assert lib.bfp_fp8_sizes(1, (1 << 23) + 1, ctypes.byref(a), ctypes.byref(b)) == E_UNSUP
    assert lib.bfp_fp8_sizes(1, 5, None, ctypes.byref(b)) == E_ARG


def test_quantize_refusals(lib):
    q = lambda x=at(0), R=10, C=300, ax=1, f=0, c=at(1), e=at(2), s=None, xt=0: lib.bfp_quantize_fp8(x, xt, R, C, ax, f, c, e, s, None)  # noqa: E731
    assert q(x=None) == q(c=None) == q(e=None) == E_ARG
    assert q(ax=2) == q(f=2) == q(f=-1) == q(R=-1) == q(C=-1) == E_ARG
    assert q(x=at(0) + 2) == q(c=at(1) + 8) == q(e=at(2) + 2) == q(s=at(3) + 1) == E_ARG
    assert q(C=(1 << 23) + 1) == E_UNSUP and q(ax=0, R=(1 << 23) + 1) == E_UNSUP
    assert q(R=1 << 31) == E_UNSUP
    # outputs over the input, or each other
    assert q(c=at(0) + 16) == q(e=at(0)) == q(c=at(1), e=at(1) + 128) == E_ARG
    assert q(xt=2) == q(xt=-1) == q(xt=1, x=at(0) + 1) == q(xt=1, c=at(0) + 5984) == E_ARG
    assert q(R=0) == q(C=0) == OK
    # launches of 2^32 threads: 32 for four blocks of a row, 256 for a tile of 128 x 128
    assert q(R=1 << 27, C=5) == q(R=1 << 25, C=2048, x=at(0)) == q(ax=0, R=1, C=1 << 31) == E_UNSUP
    d = lambda *p: lib.bfp_quantize_fp8_dual(at(0), 0, 10, 300, 0, *p, None, None)  # noqa: E731
    assert d(None, at(2), at(3), at(4)) == d(at(1), at(2), at(3), None) == E_ARG
    assert d(at(1), at(2), at(1), at(4)) == d(at(1), at(2), at(3), at(2)) == E_ARG
    v = lambda c=at(1), e=at(2), rows=10, n=300, f=0, y=at(0): lib.bfp_dequantize_fp8(c, e, rows, n, f, y, None)  # noqa: E731
    assert v(c=None) == v(y=None) == v(f=3) == v(y=at(1)) == v(rows=-1) == E_ARG
    assert v(rows=0) == v(n=0) == OK
    assert v(rows=1 << 32, n=1) == v(rows=1 << 30, n=13) == E_UNSUP


def test_gemm_refusals(lib):
    def g(a=at(0), ea=at(1), fa=0, b=at(2), eb=at(3), fm=0, M=100, N=90, K=300, C=at(4), ldc=90, ws=None, n=0, ct=0):
        return lib.bfp_gemm_fp8(a, ea, fa, b, eb, fm, M, N, K, C, ct, ldc, ws, n, None)
    assert g(a=None) == g(ea=None) == g(b=None) == g(eb=None) == g(C=None) == g(fa=2) == g(fm=-1) == E_ARG
    assert g(M=-1) == g(N=-1) == g(K=-1) == E_ARG
    assert g(a=at(0) + 4) == g(ea=at(1) + 1) == g(C=at(4) + 2) == E_ARG
    assert g(ct=2) == g(ct=1, C=at(4) + 1) == E_ARG
    assert g(ldc=89) == E_SHAPE
    assert g(K=(1 << 23) + 1) == g(M=1 << 31) == g(N=1 << 31, ldc=1 << 31) == E_UNSUP
    assert g(M=1 << 30, N=1 << 30, ldc=1 << 30) == E_UNSUP
    assert g(C=at(0)) == g(C=at(3)) == g(C=at(2) - 4) == E_ARG
    assert g(M=0) == g(N=0, ldc=0) == OK
    need, parts = ctypes.c_size_t(0), ctypes.c_int(0)
    out = [ctypes.byref(ctypes.c_int(0)) for _ in range(3)] + [ctypes.byref(parts)]
    assert lib.bfp_gemm_fp8_ws_size(100, 90, 8192, None) == E_ARG
    assert lib.bfp_gemm_fp8_ws_size(100, 90, 1 << 20, ctypes.byref(need)) == OK
    assert lib.bfp_gemm_fp8_route(100, 90, 1 << 20, need.value, *out) == OK
    assert (parts.value > 1) == (need.value > 0)
    if need.value:
        k = dict(K=1 << 20, n=need.value)
        big = 1 << 34  # (apart from everything)
        spread = dict(a=big, ea=2 * big, b=3 * big, eb=4 * big, C=5 * big)
        assert g(**spread, **k, ws=6 * big + 4) == g(**spread, **k, ws=big) == g(**spread, **k, ws=5 * big) == E_ARG
        assert lib.bfp_gemm_fp8_route(100, 90, 1 << 20, need.value - 1, *out) == OK
        assert parts.value == 1
    assert lib.bfp_gemm_fp8_route(0, 90, 100, 0, *out) == E_ARG
    # a launch has fewer than 2^32 threads, whatever the sizes
    v = [ctypes.c_int(0) for _ in range(4)]
    for M, N, K in ((1, 1 << 28, 128), (1, (1 << 31) - 64, 128), (1 << 28, 3, 1), (1 << 18, 1 << 18, 128), (16, 1 << 30, 4096)):
        if lib.bfp_gemm_fp8_route(M, N, K, 1 << 40, *map(ctypes.byref, v)) == E_UNSUP:
            continue
        rows, cols, waves, parts = (x.value for x in v)
        assert -(-M // rows) * -(-N // cols) * parts * (64 * waves if waves else 256) < 1 << 32, (M, N, K)
    assert g(M=1 << 20, N=1 << 12, ldc=1 << 12, K=0) == E_UNSUP
    assert lib.bfp_gemm_fp8_ws_size(100, 90, 0, ctypes.byref(need)) == OK and need.value == 0
    assert g(K=0, a=None, ea=None, b=None, eb=None, C=at(4) + 2) == E_ARG  # (checked, and nothing divides by K)


def test_norm_refusals(lib):
    def n(x=at(0), z=at(1), w=at(2), rows=10, d=256, eps=1e-6, h=at(3), r=at(4), y=at(5), xt=0):
        return lib.bfp_rms_norm(x, xt, z, w, rows, d, eps, h, r, y, None)
    assert n(x=None) == n(w=None) == n(y=None) == n(rows=-1) == n(d=-1) == E_ARG
    assert n(eps=-1.0) == n(eps=math.nan) == n(eps=math.inf) == E_ARG
    assert n(d=16385) == n(rows=1 << 31) == E_UNSUP
    assert n(rows=1 << 26, d=1) == n(rows=1 << 24, d=1025) == n(rows=1 << 22, d=4097) == E_UNSUP
    assert n(x=at(0) + 2) == n(h=at(3) + 1) == n(y=at(5) + 2) == E_ARG
    assert n(h=at(0) + 4) == n(h=at(1) - 4) == n(h=at(2)) == n(h=at(4)) == n(y=at(3)) == n(y=at(2)) == E_ARG
    assert n(y=at(0) + 4) == n(r=at(0)) == n(r=at(5)) == E_ARG
    assert n(h=at(0), y=at(0)) == n(h=at(1), y=at(1)) == E_ARG
    # (in place of a BF16 x would be over values that are still to be read)
    assert n(xt=2) == n(xt=1, h=at(0)) == n(xt=1, y=at(0)) == n(xt=1, x=at(0) + 1) == E_ARG
    assert n(rows=0) == n(d=0) == OK
    f = lambda fmt=0, c=at(5), e=at(6), s=None: lib.bfp_rms_norm_fp8(at(0), 0, at(1), at(2), 10, 256, 1e-6, at(3), at(4), fmt, c, e, s, None)  # noqa: E731
    assert f(fmt=2) == f(c=None) == f(e=None) == f(c=at(5) + 4) == f(s=at(7) + 2) == f(c=at(0)) == f(e=at(3)) == f(e=at(5)) == E_ARG
    b = lambda d=256, m=4, mode=0, c=at(5), e=at(6): lib.bfp_rms_norm_bfp(at(0), 0, at(1), at(2), 10, d, 1e-6, at(3), at(4), m, mode, 0, c, e, None, None)  # noqa: E731
    assert b(m=0) == b(m=9) == E_PREC
    assert b(d=250) == E_SHAPE
    assert b(mode=3) == b(c=None) == b(e=None) == b(c=at(5) + 2) == b(c=at(1)) == b(e=at(5)) == E_ARG


def test_norm_gradient_refusals(lib):
    need = ctypes.c_size_t(0)
    assert lib.bfp_rms_norm_grad_ws_size(10, 256, ctypes.byref(need)) == OK and need.value >= 4 * 256

    def g(dy=at(0), h=at(1), r=at(2), w=at(3), z=at(4), rows=10, d=256, dx=at(5), dw=at(6), ws=at(7), nb=need.value, yt=0):
        return lib.bfp_rms_norm_grad(dy, yt, h, r, w, z, rows, d, dx, dw, ws, nb, None)
    assert g(dy=None) == g(h=None) == g(r=None) == g(w=None) == g(dx=None) == g(dw=None) == g(ws=None) == E_ARG
    assert g(yt=2) == g(yt=1, dx=at(0)) == g(yt=1, dy=at(0) + 1) == E_ARG
    assert g(nb=need.value - 1) == g(rows=-1) == E_ARG
    assert g(d=16385) == E_UNSUP
    assert g(dx=at(0) + 4) == g(dx=at(4) - 4) == g(dx=at(1)) == g(dx=at(2)) == g(dx=at(3)) == E_ARG
    assert g(dw=at(0)) == g(dw=at(5)) == g(ws=at(1)) == g(ws=at(5)) == g(ws=at(6)) == E_ARG
    assert g(dw=at(6) + 2) == g(ws=at(7) + 1) == E_ARG


def test_list_refusals(lib):
    ptrs = lambda *p: (ctypes.c_void_p * len(p))(*p)  # noqa: E731
    sizes = lambda *n: (ctypes.c_int64 * len(n))(*n)  # noqa: E731
    need = ctypes.c_size_t(0)
    assert lib.bfp_sum_squares_ws_size(sizes(5, 0, 100000), 3, ctypes.byref(need)) == OK and need.value > 0
    assert lib.bfp_sum_squares_ws_size(sizes(-1), 1, ctypes.byref(need)) == E_ARG
    assert lib.bfp_sum_squares_ws_size(None, 1, ctypes.byref(need)) == E_ARG
    s = lambda p=ptrs(at(0), at(1)), n=sizes(100, 100), c=2, o=at(2), ws=at(3), nb=64, t=0: lib.bfp_sum_squares(p, t, n, c, o, ws, nb, None)  # noqa: E731
    assert s(p=ptrs(at(0), None)) == s(n=sizes(100, -1)) == s(c=-1) == s(ws=None) == s(nb=8) == E_ARG
    assert s(t=2) == s(t=1, p=ptrs(at(0), at(1) + 1)) == E_ARG
    assert s(p=ptrs(at(0), at(1) + 2)) == s(o=at(2) + 4) == s(o=at(0)) == s(ws=at(1)) == s(o=at(3)) == E_ARG

    def c(p=ptrs(at(0), at(1)), o=ptrs(at(2), at(3)), n=sizes(100, 100), k=2, m=1.0, sq=at(4), norm=at(5), t=0, sums=1):
        return lib.bfp_clip_gradients(p, o, t, n, k, m, sq, sums, norm, None)
    assert c(m=-1.0) == c(m=math.nan) == c(sq=None) == c(norm=None) == c(norm=at(4)) == c(sq=at(4) + 4) == E_ARG
    assert c(p=ptrs(at(0), None)) == c(o=ptrs(None, at(3))) == c(o=None) == E_ARG
    # the same tensor twice in place, outputs over each other or over another input
    assert c(p=ptrs(at(0), at(0)), o=ptrs(at(0), at(0))) == E_ARG
    assert c(o=ptrs(at(2), at(2) + 396)) == c(o=ptrs(at(2), at(2) - 396)) == c(o=ptrs(at(1), at(2))) == E_ARG
    assert c(o=ptrs(at(0) + 4, at(2))) == c(o=ptrs(at(2), at(0) - 4)) == c(o=ptrs(at(0), at(0))) == E_ARG
    assert c(sums=0) == c(sums=2, norm=at(4) + 8) == c(sums=2, o=ptrs(at(4) + 8, at(3))) == E_ARG and c(sums=1025) == E_UNSUP
    assert c(t=2) == c(t=1, o=ptrs(at(2), at(2) + 198)) == E_ARG
    assert c(norm=at(3)) == c(norm=at(1)) == c(sq=at(2)) == E_ARG


def test_binding_refusals():
    """Checks of arguments that come before any device work."""
    x = torch.zeros(4, 256)
    for call in (lambda: fb.quantize_fp8(x), lambda: fb.quantize_fp8_dual(x), lambda: fb.rms_norm(x, torch.ones(256)),
                 lambda: fb.rms_norm_grad(x, x, torch.ones(4), torch.ones(256)), lambda: fb.sum_squares([x]),
                 lambda: fb.clip_gradients([x], 1.0), lambda: fb.tensor_list([x])):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        fb.quantize_fp8(x, fmt="e3m4")
    with pytest.raises(ValueError):
        fb.tensor_list([])
    a, b = fb.FP8Tensor.empty(4, 256, "e4m3", "cpu"), fb.FP8Tensor.empty(4, 128, "e4m3", "cpu")
    with pytest.raises(ValueError):
        fb.gemm_fp8(a, b)
    with pytest.raises(TypeError):  # (on the host)
        fb.gemm_fp8(a, a)
    data, scales = a.data, a.scales
    for args, err in (((data.view(torch.uint8), scales, 4, 256, "e4m3"), TypeError), ((data, scales, 4, 256, "e5m2"), TypeError),
                      ((data, scales, 4, 384, "e4m3"), ValueError), ((data, scales, 5, 256, "e4m3"), ValueError),
                      ((data, scales[:, :2], 4, 256, "e4m3"), ValueError), ((data, scales.T, 4, 256, "e4m3"), ValueError),
                      ((data, scales.to(torch.int8), 4, 256, "e4m3"), TypeError)):
        with pytest.raises(err):
            fb.FP8Tensor(*args)
    assert a.codes.shape == (4, 256) and b.exp.shape == (4, 1) and b.scales.shape == (4, 4)


def test_calls_run_with_their_tensors_device_current(monkeypatch):
    """The default stream's handle is the same for every device: a call for tensors of
    another device than the current one makes it current."""
    from paper_2110_15456_amd import layer
    now, seen = [0], []

    class Device:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.old, now[0] = now[0], self.dev.index

        def __exit__(self, *e):
            now[0] = self.old

    class Lib:
        def entry(self, *args):
            seen.append((now[0], args))
            return 0
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(layer, "_current_device", lambda: now[0])
    monkeypatch.setattr(layer, "_stream", lambda dev: 0)
    monkeypatch.setattr(layer, "load", Lib)
    for index in (0, 3):
        layer._call("entry", torch.device("cuda", index), 7)
        assert seen[-1] == (index, (7, 0)) and now[0] == 0
