"""The 8-bit products, the norm and the clipping together, as a training step of a linear
layer behind a norm uses them: against the formulas in 64 bits on the same rounded
operands, captured and replayed, on two streams, and on tensors past 2^31 values."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2110_15456_amd as fb
from tests import fp8_util as F

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


class Layer:
    """y = norm(x + residual) W^T in 8 bits, its gradients, their clipping and W's update."""

    def __init__(self, d_in, d_out, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.w = torch.randn((d_out, d_in), generator=g, device=DEV) * 0.05
        self.scale = 1.0 + 0.1 * torch.randn(d_in, generator=g, device=DEV)

    def step(self, x, residual, dy, dh, lr, max_norm):
        """(y, h, gradient of x, norm, new weights, new scale)"""
        wr, wc = fb.quantize_fp8_dual(self.w)
        n, h, rstd = fb.rms_norm(x, self.scale, residual=residual, eps=EPS, save=True)
        nr, nc = fb.quantize_fp8_dual(n)
        y = fb.gemm_fp8(nr, wr, dtype=torch.bfloat16)
        gr, gc = fb.quantize_fp8_dual(dy, fmt="e5m2")
        dn = fb.gemm_fp8(gr, wc)
        dw = fb.gemm_fp8(gc, nc)
        dx, dscale = fb.rms_norm_grad(dn, h, rstd, self.scale, dresidual=dh)
        norm = fb.clip_gradients([dw, dscale], max_norm)
        w, _, _ = fb.weight_update(self.w, dw, -lr)
        return y, h, dx, norm, w, self.scale - lr * dscale


def inputs(rows, d_in, d_out, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((rows, d_in), generator=g, device=DEV).bfloat16()
    residual = torch.randn((rows, d_in), generator=g, device=DEV)
    dy = (1e-3 * torch.randn((rows, d_out), generator=g, device=DEV)).bfloat16()
    dh = 1e-3 * torch.randn((rows, d_in), generator=g, device=DEV)
    return x, residual, dy, dh


@pytest.mark.parametrize("rows,d_in,d_out", [(1, 64, 48), (200, 272, 400), (513, 1040, 336)])
def test_step_is_the_formulas(rows, d_in, d_out):
    layer, v = Layer(d_in, d_out, 1), inputs(rows, d_in, d_out, 2)
    y, h, dx, norm, w, scale = (t.double().cpu().numpy() for t in layer.step(*v, lr=0.1, max_norm=0.5))
    x, res, dy, dh = (t.double().cpu().numpy() for t in v)
    W, S = layer.w.double().cpu().numpy(), layer.scale.double().cpu().numpy()
    h64 = np.float32(x + res).astype(np.float64)
    r = 1.0 / np.sqrt((h64 * h64).mean(axis=1, keepdims=True) + EPS)
    n = np.float32(h64 * r * S)

    def both(a, fmt="e4m3"):
        a = np.float32(a)
        return (F.values(*F.quantize(a, fmt), fmt), F.values(*F.quantize(np.ascontiguousarray(a.T), fmt), fmt))

    (wr, wc), (nr, nc), (gr, gc) = both(W), both(n), both(dy, "e5m2")
    # The matrix instruction's alignment: at most 7 2^-13 of the largest |a| |b| of eight
    # products each, bounded by the rows' largest values.
    lost = lambda a, b: 7 * 2.0 ** -13 * (a.shape[1] / 8 + 1) * np.abs(a).max(axis=1)[:, None] * np.abs(b).max(axis=1)[None]  # noqa: E731
    Y = nr @ wr.T
    assert np.array_equal(h, h64)
    assert np.all(np.abs(y - Y) <= lost(nr, wr) + 2.0 ** -8 * np.abs(Y))
    dn, dw = gr @ wc.T, gc @ nc.T
    e_dn = lost(gr, wc)
    u = dn * S
    dx64 = r * u - h64 * r ** 3 * (u * h64).mean(axis=1, keepdims=True) + dh
    e_u = e_dn * np.abs(S)
    e = r * e_u + np.abs(h64) * r ** 3 * (e_u * np.abs(h64)).mean(axis=1, keepdims=True)
    size = np.abs(r * u) + np.abs(h64) * r ** 3 * np.abs(u * h64).mean(axis=1, keepdims=True) + np.abs(dh)
    assert np.all(np.abs(dx - dx64) <= e + 16 * 2.0 ** -24 * size)
    ds = (dn * h64 * r).sum(axis=0)
    N = math.sqrt((dw ** 2).sum() + (ds ** 2).sum())
    e_n = math.sqrt((lost(gc, nc) ** 2).sum() + ((e_dn * np.abs(h64) * r).sum(axis=0) ** 2).sum()) + 1e-6 * N
    assert abs(norm[0] - N) <= e_n
    f = min(1.0, 0.5 / N)
    e_f = 0.5 / N * (e_n / max(N - e_n, 1e-30)) if N + e_n > 0.5 else 0.0
    assert np.all(np.abs(w - (W - 0.1 * f * dw)) <= 0.1 * (f * lost(gc, nc) + e_f * np.abs(dw)) + 2.0 ** -22 * (np.abs(W) + np.abs(dw)))
    e_s = 0.1 * (f * (e_dn * np.abs(h64) * r).sum(axis=0) + e_f * np.abs(ds))
    assert np.all(np.abs(scale - (S - 0.1 * f * ds)) <= e_s + 2.0 ** -20 * (np.abs(S) + np.abs(ds)))


def test_step_captured_and_replayed():
    layer, a = Layer(272, 400, 1), inputs(200, 272, 400, 2)
    held = [t.clone() for t in a]
    want = [layer.step(*inputs(200, 272, 400, s), lr=0.1, max_norm=0.5) for s in (2, 3, 4)]
    layer.step(*held, lr=0.1, max_norm=0.5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.step(*held, lr=0.1, max_norm=0.5)
    for turn in range(2):
        for k, s in enumerate((2, 3, 4)):
            for t, v in zip(held, inputs(200, 272, 400, s)):
                t.copy_(v)
            graph.replay()
            torch.cuda.synchronize()
            eager = layer.step(*inputs(200, 272, 400, s), lr=0.1, max_norm=0.5)  # (between the replays)
            torch.cuda.synchronize()
            for o, w, e in zip(out, want[k], eager):
                assert torch.equal(o, w) and torch.equal(e, w)


def test_two_streams_at_once():
    layers = [Layer(1040, 336, s) for s in (1, 2)]
    data = [inputs(513, 1040, 336, s) for s in (3, 4)]
    want = [l.step(*v, lr=0.1, max_norm=0.5) for l, v in zip(layers, data)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(layers[k].step(*data[k], lr=0.1, max_norm=0.5))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[k]))


def test_conversions_and_norm_past_2_31_values():
    rows, d = (1 << 17) + 5, 16400  # 2.15e9 values
    x = torch.empty((rows, d), dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    pick = [0, 1, 65535, 131066, rows - 1]
    host = x[pick].float().cpu().numpy()
    t = fb.quantize_fp8(x)
    codes, byte = F.quantize(host, "e4m3")
    assert np.array_equal(t.data.view(torch.uint8)[pick].cpu().numpy()[:, :d], codes)
    assert np.array_equal(t.scales[pick].cpu().numpy()[:, :byte.shape[1]], byte)
    tr, tc = fb.quantize_fp8_dual(x)
    assert torch.equal(tr.data.view(torch.uint8), t.data.view(torch.uint8)) and torch.equal(tr.scales, t.scales)
    del tr, t
    cols = [0, 127, 8200, d - 1]
    codes, byte = F.quantize(np.ascontiguousarray(x[:, cols].float().cpu().numpy().T), "e4m3")
    assert np.array_equal(tc.data.view(torch.uint8)[cols].cpu().numpy()[:, :rows], codes)
    assert np.array_equal(tc.scales[cols].cpu().numpy()[:, :byte.shape[1]], byte)
    del tc, x
    torch.cuda.empty_cache()
    x = torch.empty((rows, 16384), dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(2))
    w = torch.ones(16384, device=DEV)
    res = torch.zeros((rows, 16384), device=DEV)
    y, h, r = fb.rms_norm(x, w, residual=res, h_out=res, to="e4m3", save=True)
    for i in pick:
        y1, h1, r1 = fb.rms_norm(x[i:i + 1], w, to="e4m3", save=True)
        assert torch.equal(y1.data.view(torch.uint8)[0], y.data.view(torch.uint8)[i])
        assert torch.equal(h1[0], h[i]) and torch.equal(r1[0], r[i])
    del y
    dx, _ = fb.rms_norm_grad(x, h, r, w, out=None)
    for i in pick:
        one, _ = fb.rms_norm_grad(x[i:i + 1], h[i:i + 1], r[i:i + 1], w)
        assert torch.equal(one[0], dx[i])
    del dx, h, res
    torch.cuda.empty_cache()


def test_product_of_more_than_2_31_values():
    M, N, K = 70001, 32000, 200
    g = torch.Generator(device=DEV).manual_seed(1)
    a, b = (torch.randint(-7, 8, (n, K), generator=g, device=DEV).float() for n in (M, N))
    C = fb.gemm_fp8(fb.quantize_fp8(a), fb.quantize_fp8(b), dtype=torch.bfloat16)
    for i in (0, 255, 256, 33333, 67108, M - 1):
        assert torch.equal(C[i], (a[i].double() @ b.double().t().contiguous()).bfloat16())


def test_one_list_of_far_more_tensors_than_a_launch_takes():
    n = 1000
    flat = torch.randn(n * 50, device=DEV)
    gs = list(flat.clone().split(50))
    norm = fb.clip_gradients(gs, 1.0)
    want = flat.double().norm()
    assert abs(float(norm) - float(want)) <= 1e-12 * float(want)
    got = torch.cat(gs).double()
    assert bool(((got - flat.double() / want).abs() <= 2.0 ** -23 * (flat.double() / want).abs()).all())


def test_step_with_another_device_current(monkeypatch):
    """The path that makes the tensors' device current for a call gives the same step."""
    from paper_2110_15456_amd import layer as L
    layer, v = Layer(272, 400, 1), inputs(70, 272, 400, 2)
    want = layer.step(*v, lr=0.1, max_norm=0.5)
    made = []

    class MadeCurrent(torch.cuda.device):
        def __init__(self, dev):
            made.append(dev)
            super().__init__(dev)
    monkeypatch.setattr(torch.cuda, "device", MadeCurrent)
    monkeypatch.setattr(L, "_current_device", lambda: -1)
    got = layer.step(*v, lr=0.1, max_norm=0.5)
    assert len(made) >= 10 and set(made) == {torch.device(DEV)}
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_status_words_and_other_refusals():
    x, w = torch.randn(4, 256, device=DEV), torch.ones(256, device=DEV)
    for bad in (torch.zeros(1, dtype=torch.uint8, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV),
                torch.zeros(0, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32)):
        for call in (lambda: fb.quantize_fp8(x, status=bad), lambda: fb.quantize_fp8_dual(x, status=bad),
                     lambda: fb.rms_norm(x, w, to="e4m3", status=bad), lambda: fb.rms_norm(x, w, to=4, status=bad)):
            with pytest.raises((TypeError, ValueError)):
                call()
    a = fb.quantize_fp8(x)
    host = fb.FP8Tensor(a.data.cpu(), a.scales.cpu(), 4, 256, "e4m3")
    for call in (lambda: fb.gemm_fp8(a, host), lambda: fb.gemm_fp8(host, host), lambda: fb.dequantize_fp8(host),
                 lambda: fb.quantize_fp8(x, out=host), lambda: fb.rms_norm(x, w, to="e4m3", out=host),
                 lambda: fb.gemm_fp8(a, a, out=torch.empty(4, 4, device=DEV).t()[:, :3]),
                 lambda: fb.gemm_fp8(a, a, out=torch.empty(4, 4, device=DEV)[:, ::2]),
                 lambda: fb.gemm_fp8(a, a, dtype=torch.float16)):
        with pytest.raises((TypeError, ValueError)):
            call()
    with pytest.raises(fb.BFPError):  # (a product over its own operand)
        fb.gemm_fp8(a, a, out=a.data.view(torch.float32)[:, :4])
