"""8-bit floating-point blocks on the GPU: conversions bit for bit against the CPU's
(tests/fp8_util.py), products against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2110_15456_amd as fb
from paper_2110_15456_amd import synth
from tests import fp8_util as F

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def bf16(x):
    """(x rounded to BF16 on the GPU, the same in FP32 on the CPU)"""
    t = gpu(x).bfloat16()
    return t, t.float().cpu().numpy()


def spread(shape, seed):
    """Values over many powers of two, zeros, subnormals and values at the formats' borders."""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal(shape) * 2.0 ** rng.integers(-30, 30, shape)).astype(np.float32)
    flat = x.reshape(-1)
    if flat.size:
        at = rng.integers(0, flat.size, max(1, flat.size // 16))
        flat[at] = rng.choice(np.array([0.0, -0.0, 1e-40, -1e-39, 448.0, 449.0, 1.75, 1.7500001, 2.0 ** -126, 3e38, 57344.0,
                                        1.0625, 1.1875, -1.125], np.float32), at.size)
    return x


SHAPES = [(1, 1), (1, 127), (3, 128), (2, 129), (5, 512), (7, 513), (64, 777), (129, 1050), (300, 4096), (2, 5000),
          (9, 2), (200, 3), (131, 4), (130, 5), (33, 6), (17, 7), (140, 130), (300, 131), (257, 257)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("shape", SHAPES)
def test_conversions_are_the_oracles(shape, fmt):
    print(shape, fmt, flush=True)
    for seed, x in ((1, spread(shape, 1)), (2, synth.draw("grads", shape, 2))):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        F.check_tensor(fb.quantize_fp8(gpu(x), fmt=fmt, status=st), x, fmt)
        F.check_tensor(fb.quantize_fp8(gpu(x), axis=0, fmt=fmt, status=st), np.ascontiguousarray(x.T), fmt)
        tr, tc = fb.quantize_fp8_dual(gpu(x), fmt=fmt, status=st)
        F.check_tensor(tr, x, fmt)
        F.check_tensor(tc, np.ascontiguousarray(x.T), fmt)
        assert int(st) == 0
        y = fb.dequantize_fp8(tr).cpu().numpy().astype(np.float64)
        want = F.values(*F.quantize(x, fmt), fmt)
        assert np.array_equal(y, np.float32(want).astype(np.float64))
        t, x = bf16(x)
        F.check_tensor(fb.quantize_fp8(t, fmt=fmt, status=st), x, fmt)
        F.check_tensor(fb.quantize_fp8(t, axis=0, fmt=fmt), np.ascontiguousarray(x.T), fmt)
        tr, tc = fb.quantize_fp8_dual(t, fmt=fmt)
        F.check_tensor(tr, x, fmt)
        F.check_tensor(tc, np.ascontiguousarray(x.T), fmt)
        assert bool(np.isfinite(x).all()) == (int(st) == 0)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_every_code_comes_back(fmt):
    """All finite codes at the scales' ends and in the middle, ties on either side."""
    t = F.table(fmt)
    for p in (-110, 0, 100):
        v = np.concatenate([t, -t, (t[1:] + t[:-1]) / 2, -(t[1:] + t[:-1]) / 2, np.full(128, t[-1])])
        x = np.float32(v * 2.0 ** p)
        x = np.resize(x, (6, 128))
        x[:, 0] = np.float32(t[-1] * 2.0 ** p)  # (the block's largest: the scale is 2^p)
        F.check_tensor(fb.quantize_fp8(gpu(x), fmt=fmt), x, fmt)


@pytest.mark.parametrize("n", [300, 301, 302, 303])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_infinities_and_nan(fmt, n):
    x = synth.draw("weights", (140, n), 3)
    x[3, 5], x[3, 200], x[77, 299], x[130, 0] = np.inf, -np.inf, np.nan, np.nan
    x[50, 128:256] = np.nan  # a block of nothing else
    for call in (lambda s: [(fb.quantize_fp8(gpu(x), fmt=fmt, status=s), x)],
                 lambda s: [(fb.quantize_fp8(gpu(x), axis=0, fmt=fmt, status=s), x.T)],
                 lambda s: list(zip(fb.quantize_fp8_dual(gpu(x), fmt=fmt, status=s), (x, x.T)))):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        for t, want in call(st):
            F.check_tensor(t, np.ascontiguousarray(want), fmt)
        assert int(st) == 1


def test_leading_axes_are_rows_and_empty_tensors():
    x = synth.draw("weights", (3, 4, 200), 5)
    t = fb.quantize_fp8(gpu(x))
    assert (t.rows, t.len) == (12, 200)
    F.check_tensor(t, x.reshape(12, 200), "e4m3")
    assert t.codes.shape == (12, 200) and t.exp.shape == (12, 2)
    for shape in ((0, 200), (5, 0)):
        e = torch.empty(shape, device=DEV)
        fb.quantize_fp8(e), fb.quantize_fp8(e, axis=0), fb.quantize_fp8_dual(e)
        fb.dequantize_fp8(fb.quantize_fp8(e))


def product(a, b):
    """(C, a bound of what its sums may lose) in 64 bits.  Of eight consecutive products
    the seven smaller may lose what lies below 2^-13 of the largest, which is at most the
    largest |a| times the largest |b| of the eight; sums of 64 products, of those and of
    parts lose at most a unit in the last place, 2^-23 of the sum of |terms|, each."""
    K = a.shape[1]
    pad = ((0, 0), (0, -K % 8))
    top_a, top_b = (np.abs(np.pad(v, pad)).reshape(v.shape[0], -1, 8).max(axis=2) for v in (a, b))
    return a @ b.T, 7 * 2.0 ** -13 * (top_a @ top_b.T) + (K / 64 + 16) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)


PRODUCTS = [(1, 1, 1), (1, 16, 128), (16, 100, 4096), (17, 777, 1050), (33, 65, 129), (64, 64, 8192), (130, 257, 640),
            (300, 511, 384), (1531, 777, 1050), (2, 3000, 513), (700, 5, 5000), (1024, 1024, 256), (2049, 1100, 1000),
            (8, 1, 30000), (513, 1025, 2100)]


@pytest.mark.parametrize("fmt_a,fmt_b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_products(M, N, K, fmt_a, fmt_b):
    print(M, N, K, fmt_a, fmt_b, flush=True)
    a, b = synth.draw("half_normal", (M, K), 1), synth.draw("grads", (N, K), 2)
    A, B = fb.quantize_fp8(gpu(a), fmt=fmt_a), fb.quantize_fp8(gpu(b), fmt=fmt_b)
    C, most = product(F.values(*F.quantize(a, fmt_a), fmt_a), F.values(*F.quantize(b, fmt_b), fmt_b))
    for ws in (True, False):
        got = fb.gemm_fp8(A, B, workspace=ws).cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - C) <= most)
    got = fb.gemm_fp8(A, B)
    assert torch.equal(fb.gemm_fp8(A, B), got)
    assert torch.equal(fb.gemm_fp8(A, B, dtype=torch.bfloat16), got.bfloat16())


@pytest.mark.parametrize("fmt_a,fmt_b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_products_of_small_integers_are_exact(M, N, K, fmt_a, fmt_b):
    """Integers up to 7, with scales of their own for every block of every row, all within
    two powers of two: exact in any order and alignment, so a value in a wrong place, or a
    wrong scale, shows."""
    rng = np.random.default_rng(K)

    def draw(rows, fmt):
        v = rng.integers(-7, 8, (rows, K)).astype(np.float64)
        t = fb.FP8Tensor.empty(rows, K, fmt, DEV)
        e = rng.integers(126, 129, tuple(t.scales.shape)).astype(np.uint8)
        codes = np.zeros(tuple(t.data.shape), np.uint8)
        codes[:, :K] = np.searchsorted(F.table(fmt), np.abs(v)) | np.where(v < 0, 0x80, 0)
        t.data.view(torch.uint8).copy_(gpu(codes))
        t.scales.copy_(gpu(e))
        return t, v * np.repeat(2.0 ** (e.astype(np.float64) - 127), 128, axis=1)[:, :K]

    (A, a), (B, b) = draw(M, fmt_a), draw(N, fmt_b)
    C = a @ b.T
    for ws in (True, False):
        got = fb.gemm_fp8(A, B, workspace=ws).cpu().numpy().astype(np.float64)
        assert np.array_equal(got, C)


def test_output_slices_rows_behind_and_no_k():
    a, b = synth.draw("weights", (37, 300), 1), synth.draw("weights", (50, 300), 2)
    A, B = fb.quantize_fp8(gpu(a)), fb.quantize_fp8(gpu(b))
    want = fb.gemm_fp8(A, B)
    wide = torch.full((40, 77), 7.0, device=DEV)
    fb.gemm_fp8(A, B, out=wide[1:38, 3:53])
    assert torch.equal(wide[1:38, 3:53], want)
    wide[1:38, 3:53] = 7.0
    assert bool((wide == 7.0).all())  # nothing outside the slice was written
    wide = torch.full((40, 77), 7.0, device=DEV, dtype=torch.bfloat16)
    fb.gemm_fp8(A, B, out=wide[1:38, 3:53])
    assert torch.equal(wide[1:38, 3:53], want.bfloat16())
    wide[1:38, 3:53] = 7.0
    assert bool((wide == 7.0).all())
    e = torch.full((37, 50), 3.0, device=DEV)
    fb.gemm_fp8(fb.quantize_fp8(torch.empty((37, 0), device=DEV)), fb.quantize_fp8(torch.empty((50, 0), device=DEV)), out=e)
    assert not bool(e.any())
    assert fb.gemm_fp8(fb.quantize_fp8(torch.empty((0, 300), device=DEV)), B).shape == (0, 50)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(300, 511, 700), (1100, 1301, 1024), (2300, 2201, 640)])
def test_output_slices_of_large_products(M, N, K, dtype):
    A, B = (fb.quantize_fp8(gpu(synth.draw("weights", (r, K), r))) for r in (M, N))
    want = fb.gemm_fp8(A, B, dtype=dtype)
    wide = torch.full((M + 3, N + 20), 7.0, device=DEV, dtype=dtype)
    for at in (1, 3, 8):
        fb.gemm_fp8(A, B, out=wide[1:M + 1, at:at + N])
        assert torch.equal(wide[1:M + 1, at:at + N], want)
        wide[1:M + 1, at:at + N] = 7.0
        assert bool((wide == 7.0).all())


def test_nan_stays_in_its_row():
    a, b = synth.draw("weights", (70, 300), 1), synth.draw("weights", (80, 300), 2)
    B = fb.quantize_fp8(gpu(b))
    want = fb.gemm_fp8(fb.quantize_fp8(gpu(a)), B)
    a[33, 130] = np.nan
    got = fb.gemm_fp8(fb.quantize_fp8(gpu(a)), B)
    assert bool(torch.isnan(got[33]).all())
    keep = [i for i in range(70) if i != 33]
    assert torch.equal(got[keep], want[keep])


def test_given_workspace_and_another_stream():
    a, b = synth.draw("weights", (130, 8192), 1), synth.draw("weights", (100, 8192), 2)
    A, B = fb.quantize_fp8(gpu(a)), fb.quantize_fp8(gpu(b))
    want = fb.gemm_fp8(A, B)
    need = fb.gemm_fp8_ws_size(A, B)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = fb.gemm_fp8(A, B, workspace=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    assert bool((ws[need:] == 255).all())
