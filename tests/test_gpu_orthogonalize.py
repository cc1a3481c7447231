"""The orthogonalised update against its formula in 64 bits.

Tolerance, fixed before the first run: the kernels hold operands in 22 bits where
FP32 has 24 and add in FP32, so their error may be four times (2^2) that of the
same formula evaluated in FP32 on the same input, in the 2-norm of the whole
matrix; 2^-22, one rounding of the result's operands, comes on top (small matrices,
whose FP32 evaluation can be exact by chance).  The momentum has one rounding for
the product and one for the sum.
"""
from __future__ import annotations

import pytest
import torch

import paper_2110_15456_amd as fb
from gpu_util import announce

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315


def plain(u, steps=5, eps=1e-7):
    """The iteration on one matrix, in its type."""
    x = u / (u.norm() + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    for _ in range(steps):
        s = x @ x.t()
        x = A * x + (B * s + C * (s @ s)) @ x
    return x.t() if flip else x


def check(out, u, steps=5):
    want = plain(u.double(), steps)
    low = plain(u.float(), steps).double()
    norm = float(want.norm())
    assert float((out.to(want.device).double() - want).norm()) <= 4 * float((low - want).norm()) + 2.0 ** -22 * norm
    return want


SHAPES = [(1, 1), (1, 40), (40, 1), (2, 3), (31, 33), (32, 32), (33, 31), (64, 576), (100, 300), (129, 127),
          (257, 640), (640, 257), (300, 1100), (1000, 520)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", ["noise", "strong", "rank"])
def test_against_formula(rows, cols, kind):
    """Noise; a few strong directions over noise; and two directions alone, whose
    other singular values are zero."""
    announce("orthogonalize %d x %d, %s" % (rows, cols, kind))
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    r = min(2, rows, cols)
    low = torch.randn((rows, r), generator=g) @ torch.randn((r, cols), generator=g)
    noise = 1e-4 * torch.randn((rows, cols), generator=g)
    u = noise if kind == "noise" else 1e-2 * low + noise if kind == "strong" else low
    out = fb.orthogonalize(u.cuda())
    want = check(out, u)
    if kind == "noise" and min(rows, cols) * 4 <= max(rows, cols):  # (well away from zero singular values)
        s = torch.linalg.svdvals(want)
        assert 0.6 < float(s.min()) and float(s.max()) < 1.25


@pytest.mark.parametrize("shape", [(40, 300, 500), (1, 2304, 6000), (1, 6000, 2304), (2, 2300, 5000), (1, 2050, 2050),
                                   (1, 4100, 4200)])
@pytest.mark.parametrize("kind", ["noise", "strong"])
def test_large(shape, kind):
    """Many tiles: whole rounds of them, parts of K, large tiles with ragged ends.
    (The formula on the GPU, by torch's products of 64 and 32 bits.)"""
    announce("orthogonalize %d x %d x %d, %s" % (*shape, kind))
    g = torch.Generator(device="cuda").manual_seed(shape[1])
    u = 1e-4 * torch.randn(shape, generator=g, device="cuda")
    if kind == "strong":
        u += 1e-2 * (torch.randn((*shape[:2], 2), generator=g, device="cuda") @
                     torch.randn((shape[0], 2, shape[2]), generator=g, device="cuda"))
    out = fb.orthogonalize(u)
    for i in sorted({0, shape[0] // 2, shape[0] - 1}):
        check(out[i], u[i])


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_steps(steps):
    announce("orthogonalize, %d steps" % steps)
    u = torch.randn((96, 200), generator=torch.Generator().manual_seed(1))
    check(fb.orthogonalize(u.cuda(), steps=steps), u, steps)


@pytest.mark.parametrize("shape", [(3, 70, 130), (2, 2, 200, 48), (5, 33, 35)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_momentum(shape, nesterov):
    announce("orthogonal update %s" % (shape,))
    g = torch.Generator().manual_seed(7)
    grad, mom = torch.randn(shape, generator=g), 3 * torch.randn(shape, generator=g)
    gd, md = grad.cuda(), mom.cuda()
    up, new = fb.orthogonal_update(gd, md, beta=0.9, nesterov=nesterov)
    want = 0.9 * mom.double() + grad.double()  # (0.9 is passed as FP32: one more rounding of the product)
    err = (new.cpu().double() - want).abs()
    assert bool((err <= 2.0 ** -24 * (2 * (0.9 * mom).abs() + want.abs()) * 1.001).all())
    assert torch.equal(md.cpu(), mom) and torch.equal(gd.cpu(), grad)
    n32 = new.cpu()
    u = grad + torch.tensor(0.9) * n32 if nesterov else n32
    flat, got = u.reshape(-1, *shape[-2:]), up.reshape(-1, *shape[-2:])
    for i in range(flat.shape[0]):
        check(got[i], flat[i])
    # in place, with a workspace kept
    ws = torch.empty(fb.orthogonalize_ws_size(gd), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(gd)
    for _ in range(2):
        m2 = md.clone()
        up2, new2 = fb.orthogonal_update(gd, m2, beta=0.9, nesterov=nesterov, momentum_out=m2, out=out, workspace=ws)
        assert new2 is m2 and torch.equal(m2, new) and torch.equal(up2, up)


def test_scale_zeros_and_poison():
    """The size of a gradient does not matter down to values whose squares vanish in
    FP32; zeros give zeros; a matrix with a NaN or infinity spoils itself alone."""
    announce("orthogonalize scales, zeros and NaN")
    u = torch.randn((4, 48, 130), generator=torch.Generator().manual_seed(3)).cuda()
    want = fb.orthogonalize(u, eps=0.0)
    for k in (-100, 60):
        assert torch.equal(fb.orthogonalize(u * 2.0 ** k, eps=0.0), want)
    u[1] = 0.0
    u[2, 5, 7] = float("nan")
    u[3, 0, 0] = float("inf")
    out = fb.orthogonalize(u)
    check(out[0], u[0].cpu())
    assert not bool(out[1].any()) and not bool(out[2].isfinite().all()) and not bool(out[3].isfinite().all())


@pytest.mark.parametrize("power", [-124, -60, 100])
def test_far_scales(power):
    """Gradients whose norm, or the factor that normalises them, is near the ends of
    FP32's range (the smallest entries here are still normal numbers)."""
    announce("orthogonalize at 2^%d" % power)
    u = torch.randn((40, 60), generator=torch.Generator().manual_seed(9))
    u = torch.where(u.abs() < 0.25, torch.ones_like(u), u).cuda()
    assert torch.equal(fb.orthogonalize(u * 2.0 ** power, eps=0.0), fb.orthogonalize(u, eps=0.0))


def test_transposed_and_unaligned():
    """The update of the transpose is the update's transpose (the same products), and
    rows that start off a 16-byte boundary give the same bits."""
    announce("orthogonalize transposed and unaligned")
    u = torch.randn((75, 140), generator=torch.Generator().manual_seed(4)).cuda()
    out = fb.orthogonalize(u)
    assert torch.equal(fb.orthogonalize(u.t().contiguous()).t(), out)
    flat = torch.zeros(75 * 140 + 1, device="cuda")
    v = flat[1:].view(75, 140)
    v.copy_(u)
    assert torch.equal(fb.orthogonalize(v), out)


def test_graph():
    announce("orthogonal update in a graph")
    grad = torch.zeros((2, 200, 330), device="cuda")
    mom = torch.zeros_like(grad)

    def update():
        return fb.orthogonal_update(grad, mom)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        update()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = update()
    for _ in range(4):
        grad.normal_()
        mom.normal_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, update()):
            assert torch.equal(a, b)


def test_refusals():
    u = torch.zeros((8, 16), device="cuda")
    with pytest.raises(TypeError):
        fb.orthogonalize(u.cpu())
    with pytest.raises(TypeError):
        fb.orthogonalize(u.double())
    with pytest.raises(ValueError):
        fb.orthogonalize(u[0])
    with pytest.raises(ValueError):
        fb.orthogonalize(u.t())
    with pytest.raises(ValueError):
        fb.orthogonalize(u, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        fb.orthogonal_update(u, torch.zeros((16, 8), device="cuda"))
    for bad in (dict(steps=0), dict(steps=17), dict(eps=-1.0), dict(eps=float("nan")), dict(out=u)):
        with pytest.raises(fb.BFPError):
            fb.orthogonalize(u, **bad)
    with pytest.raises(fb.BFPError):
        fb.orthogonal_update(u, torch.zeros_like(u), momentum_out=u)
    assert fb.orthogonalize(torch.zeros((0, 8, 16), device="cuda")).shape == (0, 8, 16)
