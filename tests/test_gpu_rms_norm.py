"""The root-mean-square norm on the GPU: outputs against the formula in 64 bits, converted
ones byte for byte against the conversion of the FP32 output; gradients against the
formula's and against differences."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2110_15456_amd as fb
from tests import fp8_util as F

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


def gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV)


def inputs(rows, d, seed):
    rng = np.random.default_rng(seed)
    strong = np.where(rng.random(d) < 0.02, 20.0, 1.0)
    x, z = (np.float32(rng.standard_normal((rows, d)) * strong) for _ in range(2))
    return x, z, np.float32(1.0 + 0.1 * rng.standard_normal(d))


def formula(h, w, eps=EPS):
    h = h.astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):  # (a row of zeros with eps 0)
        r = 1.0 / np.sqrt((h * h).sum(axis=1, keepdims=True) / h.shape[1] + eps)
        return h * r * w.astype(np.float64), r[:, 0]


# FP32's rounding of the formula's value, and another place where 64 bits round to its border
ONE = 2.0 ** -24 * (1 + 1e-6)
SHAPES = [(1, 1), (3, 3), (1, 16), (5, 255), (2, 256), (4, 257), (7, 777), (3, 1024), (2, 1025), (33, 2048), (2, 4095),
          (64, 4096), (3, 4097), (2, 8200), (2, 8208), (3, 12288), (2, 12290), (2, 16384), (1, 16383)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,d", SHAPES)
def test_norm(rows, d, residual):
    print(rows, d, residual, flush=True)
    x, z, w = inputs(rows, d, d)
    y, h, rstd = fb.rms_norm(gpu(x), gpu(w), residual=gpu(z) if residual else None, eps=EPS, save=True)
    want_h = x + z if residual else x
    assert np.array_equal(h.cpu().numpy(), want_h)
    want, r = formula(want_h, w)
    assert np.all(np.abs(y.cpu().numpy() - want) <= ONE * np.abs(want))
    assert np.all(np.abs(rstd.cpu().numpy() - r) <= ONE * r)
    # converted on the way
    for fmt in ("e4m3", "e5m2"):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        t, h2, none = fb.rms_norm(gpu(x), gpu(w), residual=gpu(z) if residual else None, eps=EPS, to=fmt, status=st)
        assert none is None and torch.equal(h2, h) and int(st) == 0
        F.check_tensor(t, y.cpu().numpy(), fmt)
    if d % 16 == 0:
        for m in (1, 2, 3, 4, 5, 6, 7, 8):
            for rounding in ("nearest", "stochastic", "truncate"):
                t, _, _ = fb.rms_norm(gpu(x), gpu(w), residual=gpu(z) if residual else None, eps=EPS, to=m,
                                      rounding=rounding, seed=m)
                u = fb.quantize(y, m=m, rounding=rounding, seed=m)
                assert torch.equal(t.mant, u.mant) and torch.equal(t.exp, u.exp), (m, rounding)


@pytest.mark.parametrize("rows,d", SHAPES)
def test_bf16_is_its_fp32(rows, d):
    """A BF16 x or dy gives what the same values in FP32 do."""
    x, z, w = inputs(rows, d, d + 5)
    b = gpu(x).bfloat16()
    for res in (None, gpu(z)):
        for to in (None, "e4m3") + ((4,) if d % 16 == 0 else ()):
            y, h, r = fb.rms_norm(b, gpu(w), residual=res, to=to, save=True)
            y2, h2, r2 = fb.rms_norm(b.float(), gpu(w), residual=res, to=to, save=True)
            assert h.dtype == torch.float32 and torch.equal(h, h2) and torch.equal(r, r2)
            if to is None:
                assert y.dtype == torch.float32 and torch.equal(y, y2)
            else:
                p, q = ((t.data.view(torch.uint8), t.scales) if to == "e4m3" else (t.mant, t.exp) for t in (y, y2))
                assert all(torch.equal(u, v) for u, v in zip(p, q))
        dx, dw = fb.rms_norm_grad(b, h, r, gpu(w), dresidual=res)
        dx2, dw2 = fb.rms_norm_grad(b.float(), h, r, gpu(w), dresidual=res)
        assert dx.dtype == torch.float32 and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    assert fb.rms_norm(b, gpu(w))[1] is b


def test_many_rows_equal_themselves_alone():
    x, z, w = inputs(9000, 130, 1)
    y, h, r = fb.rms_norm(gpu(x), gpu(w), residual=gpu(z), save=True)
    for i in (0, 4999, 8999):
        y1, h1, r1 = fb.rms_norm(gpu(x[i:i + 1]), gpu(w), residual=gpu(z[i:i + 1]), save=True)
        assert torch.equal(y1[0], y[i]) and torch.equal(h1[0], h[i]) and torch.equal(r1[0], r[i])


def test_in_place_and_leading_axes():
    x, z, w = inputs(6, 300, 2)
    want, want_h, _ = fb.rms_norm(gpu(x), gpu(w), residual=gpu(z))
    a, b = gpu(x), gpu(z)
    y, h, _ = fb.rms_norm(a, gpu(w), residual=b, h_out=b)
    assert h is b and torch.equal(b, want_h) and torch.equal(y, want) and torch.equal(a, gpu(x))
    a, b = gpu(x), gpu(z)
    y, h, _ = fb.rms_norm(a, gpu(w), residual=b, h_out=b, out=a)
    assert y is a and torch.equal(a, want) and torch.equal(b, want_h)
    y, h, r = fb.rms_norm(gpu(x).view(2, 3, 300), gpu(w), residual=gpu(z).view(2, 3, 300), save=True)
    assert y.shape == (2, 3, 300) and torch.equal(y.view(6, 300), want) and r.shape == (6,)
    t, _, _ = fb.rms_norm(gpu(x).view(2, 3, 300), gpu(w), residual=gpu(z).view(2, 3, 300), to="e4m3")
    assert (t.rows, t.len) == (6, 300)


@pytest.mark.parametrize("rows,d", [(1, 3), (6, 300), (5, 4096), (2, 9001)])
@pytest.mark.parametrize("save", [False, True])
def test_in_place_without_a_residual_keeps_h(rows, d, save):
    """y over x: h is still what x was, and the gradients are those of a norm elsewhere."""
    x, _, w = inputs(rows, d, 12)
    dy = gpu(np.random.default_rng(6).standard_normal((rows, d)))
    want, want_h, want_r = fb.rms_norm(gpu(x), gpu(w), save=True)
    a = gpu(x)
    y, h, r = fb.rms_norm(a, gpu(w), out=a, save=save)
    assert y is a and torch.equal(a, want) and torch.equal(h, gpu(x)) and (r is not None) == save
    if save:
        assert torch.equal(r, want_r)
        for p, q in zip(fb.rms_norm_grad(dy, h, r, gpu(w)), fb.rms_norm_grad(dy, want_h, want_r, gpu(w))):
            assert torch.equal(p, q)
    a = gpu(x)
    y, h, _ = fb.rms_norm(a, gpu(w), out=a.view(rows, d), save=save)  # (another tensor on the same memory)
    assert torch.equal(a, want) and torch.equal(h, gpu(x))
    mine = torch.empty((rows, d), device=DEV)
    y, h, _ = fb.rms_norm(gpu(x), gpu(w), out=mine, save=save)
    assert y is mine and torch.equal(mine, want) and torch.equal(h, gpu(x))


def test_far_values_zeros_and_empty():
    x, _, w = inputs(8, 200, 3)
    x[0], x[1], x[2], x[3] = 0.0, x[1] * np.float32(1e30), x[2] * np.float32(1e-30), 1e-42
    for eps in (EPS, 0.0):
        rows = [1, 2, 4, 5] if eps == 0.0 else [0, 1, 2, 3, 4]
        y = fb.rms_norm(gpu(x), gpu(w), eps=eps)[0].cpu().numpy()
        want, _ = formula(x, w, eps)
        # (results below FP32's normal range: half its least step)
        assert np.all(np.abs(y[rows] - want[rows]) <= ONE * np.abs(want[rows]) + 2.0 ** -150)
    for shape in ((0, 200), (4, 0)):
        e = torch.empty(shape, device=DEV)
        ww = torch.ones(shape[1], device=DEV)
        for to in (None, "e4m3", 4) if shape[1] % 16 == 0 else (None, "e4m3"):
            fb.rms_norm(e, ww, to=to)


def test_nan_stays_in_its_row():
    x, z, w = inputs(5, 256, 4)
    want = fb.rms_norm(gpu(x), gpu(w), to="e4m3")[0]
    x[2, 7] = np.inf
    x[3, 9] = np.nan
    for to in ("e4m3", 4):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        t, _, _ = fb.rms_norm(gpu(x), gpu(w), to=to, status=st)
        assert int(st) == 1
        if to == "e4m3":
            for i in (0, 1, 4):
                assert torch.equal(t.data.view(torch.uint8)[i], want.data.view(torch.uint8)[i])
            assert bool(torch.isnan(t.codes[3].float()).all())
    y = fb.rms_norm(gpu(x), gpu(w))[0]
    assert bool(torch.isnan(y[3]).all()) and not bool(torch.isnan(y[[0, 1, 4]]).any())


def gradient(dy, h, w, dres, eps=EPS):
    """dx, dw and the sums of |terms| that their roundings are relative to, in 64 bits."""
    dy, h, w = (v.astype(np.float64) for v in (dy, h, w))
    d = h.shape[1]
    r = 1.0 / np.sqrt((h * h).sum(axis=1, keepdims=True) / d + eps)
    u = dy * w
    c = (u * h).sum(axis=1, keepdims=True) / d
    dx = r * u - h * r ** 3 * c
    S = np.abs(r * u) + np.abs(h) * r ** 3 * (np.abs(u * h).sum(axis=1, keepdims=True) / d)
    if dres is not None:
        dx, S = dx + dres, S + np.abs(dres)
    return dx, (dy * h * r).sum(axis=0), S, np.abs(dy * h * r).sum(axis=0)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,d", SHAPES + [(700, 1155), (2000, 48), (5000, 7), (4101, 260), (1030, 8300), (8, 1000), (9, 1024), (4, 5000)])
def test_gradient(rows, d, residual):
    print(rows, d, residual, flush=True)
    x, z, w = inputs(rows, d, d + 1)
    dy = np.float32(np.random.default_rng(d).laplace(0, 1e-4, (rows, d)))
    z = np.float32(z * 1e-4) if residual else None
    _, h, rstd = fb.rms_norm(gpu(x), gpu(w), eps=EPS, save=True)
    dx, dw = fb.rms_norm_grad(gpu(dy), h, rstd, gpu(w), dresidual=gpu(z) if residual else None)
    want_dx, want_dw, S, Sw = gradient(dy, x, w, z)
    # dx: rstd three times and each product and sum rounded once, at most 12 half units; four
    # terms of a row's sum are chained
    assert np.all(np.abs(dx.cpu().numpy() - want_dx) <= 16 * 2.0 ** -24 * S)
    # dw: rstd, two products, a share's sum and the result
    assert np.all(np.abs(dw.cpu().numpy() - want_dw) <= 6 * 2.0 ** -24 * Sw + 1e-45)
    again = fb.rms_norm_grad(gpu(dy), h, rstd, gpu(w), dresidual=gpu(z) if residual else None)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    # in place of dy, and of the residual path's gradient
    g = gpu(dy)
    assert torch.equal(fb.rms_norm_grad(g, h, rstd, gpu(w), dresidual=gpu(z) if residual else None, out=g)[0], dx)
    if residual:
        g = gpu(z)
        assert torch.equal(fb.rms_norm_grad(gpu(dy), h, rstd, gpu(w), dresidual=g, out=g)[0], dx)


@pytest.mark.parametrize("scale", [1e-28, 1e-18, 1e18, 1e30])
def test_gradient_of_far_values(scale):
    """h whose square, or whose r^3, leaves FP32's range (bounds as above; with eps 0)."""
    x, z, w = inputs(9, 300, 11)
    x = x * np.float32(scale)
    dy = np.float32(np.random.default_rng(3).laplace(0, 1e-4, x.shape))
    _, h, rstd = fb.rms_norm(gpu(x), gpu(w), eps=0.0, save=True)
    dx, dw = fb.rms_norm_grad(gpu(dy), h, rstd, gpu(w))
    want_dx, want_dw, S, Sw = gradient(dy, x, w, None, eps=0.0)
    # (below FP32's normal range: a unit of its least step for each of the two terms' roundings)
    assert np.all(np.abs(dx.cpu().numpy() - want_dx) <= 16 * 2.0 ** -24 * S + 2.0 ** -148)
    assert np.all(np.abs(dw.cpu().numpy() - want_dw) <= 6 * 2.0 ** -24 * Sw + 1e-45)


@pytest.mark.parametrize("d", [4, 64, 1024, 4096, 8200, 16384])
def test_sums_along_a_row_are_64_bits(d):
    """Terms 2^24, 1, -2^24, 0 over and over, with h, r and the weights 1: their mean is 1/4,
    of which sums of any four in FP32 leave 0."""
    dy = np.float32(np.tile([2.0 ** 24, 1.0, -(2.0 ** 24), 0.0], d // 4))[None].repeat(3, axis=0)
    one = torch.ones(d, device=DEV)
    _, h, rstd = fb.rms_norm(torch.ones((3, d), device=DEV), one, eps=0.0, save=True)
    assert bool((rstd == 1.0).all())
    dx, dw = fb.rms_norm_grad(gpu(dy), h, rstd, one)
    want = dy.astype(np.float64) - 0.25
    # (r, u, n, the mean and their product are exact; dx is rounded once)
    assert np.all(np.abs(dx.cpu().numpy() - want) <= 2.0 ** -24 * np.abs(want))
    assert np.array_equal(dw.cpu().numpy(), 3 * dy[0])


@pytest.mark.parametrize("rms,dy_scale", [(4e-39, 1e-4), (2.5e38, 1e30)])
def test_gradient_at_the_ends_of_rstds_range(rms, dy_scale):
    rng = np.random.default_rng(12)
    x = np.float32(rng.choice([-1.0, 1.0], (7, 300)) * rng.uniform(0.8, 1.2, (7, 300)) * rms)
    w = np.float32(1.0 + 0.1 * rng.standard_normal(300))
    dy = np.float32(rng.standard_normal(x.shape) * dy_scale)
    _, h, rstd = fb.rms_norm(gpu(x), gpu(w), eps=0.0, save=True)
    _, r = formula(x, w, 0.0)
    off = np.maximum(2.0 ** -24 * r, 2.0 ** -150) * (1 + 1e-6)  # (half of rstd's last place)
    assert np.all(np.abs(rstd.cpu().numpy() - r) <= off)
    dx, dw = fb.rms_norm_grad(gpu(dy), h, rstd, gpu(w))
    want_dx, want_dw, S, Sw = gradient(dy, x, w, None, eps=0.0)
    # test_gradient's bounds, and rstd's own error where it enters: once in r u, three times
    # in the other term, once in dw
    far = 3 * (off / r)[:, None]
    assert np.all(np.abs(dx.cpu().numpy() - want_dx) <= (16 * 2.0 ** -24 + far) * S)
    assert np.all(np.abs(dw.cpu().numpy() - want_dw) <= (6 * 2.0 ** -24 + far.max()) * Sw)


def test_no_values_in_a_row():
    """The mean of nothing is NaN, its gradient nothing."""
    e, w = torch.empty((4, 0), device=DEV), torch.ones(0, device=DEV)
    y, h, rstd = fb.rms_norm(e, w, save=True)
    assert y.shape == (4, 0) and h.shape == (4, 0) and bool(torch.isnan(rstd).all()) and rstd.shape == (4,)
    dx, dw = fb.rms_norm_grad(e, h, rstd, w)
    assert dx.shape == (4, 0) and dw.shape == (0,)


def test_gradient_against_differences():
    """Central differences of sum(dy y) of the formula in 64 bits along random directions."""
    rng = np.random.default_rng(7)
    rows, d = 6, 50
    x, _, w = inputs(rows, d, 9)
    dy = np.float32(rng.standard_normal((rows, d)))
    _, h, rstd = fb.rms_norm(gpu(x), gpu(w), eps=EPS, save=True)
    dx, dw = (v.cpu().numpy().astype(np.float64) for v in fb.rms_norm_grad(gpu(dy), h, rstd, gpu(w)))
    f = lambda a, b: (formula(a, b)[0] * dy).sum()  # noqa: E731
    for _ in range(5):
        v, u, t = rng.standard_normal((rows, d)), rng.standard_normal(d), 1e-4
        x64, w64 = x.astype(np.float64), w.astype(np.float64)
        diff = (f(x64 + t * v, w64) - f(x64 - t * v, w64)) / (2 * t)
        assert abs((dx * v).sum() - diff) <= 1e-5 * np.abs(dx * v).sum()
        diff = (f(x64, w64 + t * u) - f(x64, w64 - t * u)) / (2 * t)
        assert abs((dw * u).sum() - diff) <= 1e-5 * np.abs(dw * u).sum()


def test_gradient_of_no_rows():
    w = torch.ones(40, device=DEV)
    dx, dw = fb.rms_norm_grad(torch.empty((0, 40), device=DEV), torch.empty((0, 40), device=DEV),
                              torch.empty(0, device=DEV), w)
    assert dx.shape == (0, 40) and not bool(dw.any())
