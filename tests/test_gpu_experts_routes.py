"""The products of experts on every kernel and tile that their prices choose, in
every operand format, against products in 64 bits.

Sizes are looked for: the smallest of a grid that the library says it runs on the
kernel that a test wants, so that other prices lead to other sizes and not to
kernels that no test runs.  Values come from the definition of the conversion in
64 bits (groups of 16, nearest: half a unit added, the fraction dropped, at most
2^m - 1).  Tolerance, fixed before the first run: the library's contract for every
product, 1e-6 of the sum over groups of |their exact sum|."""
from __future__ import annotations

import ctypes
import functools
import itertools

import numpy as np
import pytest
import torch

import paper_2110_15456_amd as fb
from experts_util import plan as plain_plan
from experts_util import routing
from gpu_util import announce

pytestmark = pytest.mark.gpu

WIDTHS = [2, 4, 6, 8]
FORMATS = [(a, a, b) for a in WIDTHS for b in WIDTHS] + [(6, 4, 2), (6, 4, 6), (8, 4, 4), (8, 4, 8)]  # stored, used; of W
LARGE_IS_128 = {(6, 8), (8, 6), (8, 8)}  # two planes of each, not both FP4 codes: no other tile fits the LDS
ONE_PLANE = (2, 4)
ODD = (37, 261, 515, 1031, 2055, 4101)      # N: rows of C of any alignment, ragged last columns
LINES = (32, 256, 512, 1024, 2048, 4096)    # and rows of whole lines


# ---- sizes that take a kernel -------------------------------------------------


def rows_route(m_a, u_a, m_b, experts, slots, N, K):
    """(rows, waves) of bfp_gemm_experts_route."""
    out = [ctypes.c_int(-9), ctypes.c_int(-9)]
    assert fb.load().bfp_gemm_experts_route(m_a, m_b, experts, slots, N, K, u_a, m_b, *map(ctypes.byref, out)) == 0
    return out[0].value, out[1].value


def grad_route(m_a, m_b, experts, M, N, places):
    out = ctypes.c_int(-9)
    assert fb.load().bfp_gemm_experts_grad_route(m_a, m_b, experts, M, N, places, m_a, m_b, ctypes.byref(out)) == 0
    return out.value


@functools.lru_cache(maxsize=None)
def sizes_for(m_a, u_a, m_b, want, ks, ns=ODD):
    """The smallest (experts, slots, N, K) that runs on `want`: (rows, waves or None)."""
    grid = itertools.product((3, 5), (20, 90, 300, 700, 1500, 2900, 5500, 9000), ns, ks)
    for experts, slots, N, K in sorted(grid, key=lambda c: c[1] * c[2] * c[3]):
        rows, waves = rows_route(m_a, u_a, m_b, experts, slots, N, K)
        if rows == want[0] and want[1] in (None, waves):
            return experts, slots, N, K
    return None


def grad_sizes_for(m_a, m_b, want):
    """The smallest (experts, tokens, M, N) whose gradient runs on the tile `want`."""
    grid = itertools.product((3, 5), (600, 2300, 5000), (144, 528, 2064, 4112), (80, 272, 1040, 2064, 4112))
    for experts, tokens, M, N in sorted(grid, key=lambda c: c[0] * c[2] * c[3] * c[1]):
        places = -(-(tokens + 127 * experts) // 128) * 128 - 128
        if all(grad_route(m_a, m_b, experts, M, N, p) == want for p in (places, places + 128)):
            return experts, tokens, M, N
    return None


# ---- values in 64 bits --------------------------------------------------------


def bfp64(x, m, used=None):
    """The values of x [rows, len] in BFP at m bits, the low m - used of them dropped."""
    v = x.double().reshape(-1, 16)
    top = v.abs().amax(dim=1, keepdim=True)
    unit = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - m), torch.ones_like(top))
    q = torch.clamp(torch.floor(v.abs() / unit + 0.5), max=2 ** m - 1)
    low = 2 ** (m - (used or m))
    return (torch.sign(v) * torch.floor(q / low) * low * unit).reshape(x.shape)


def product(a, b):
    """a b^T and the sum over groups of |their sums|, for a [M, K] and b [N, K]."""
    total = torch.zeros((a.shape[0], b.shape[0]), dtype=torch.float64, device=a.device)
    size = torch.zeros_like(total)
    for k in range(0, a.shape[1], 16):
        t = a[:, k:k + 16].contiguous() @ b[:, k:k + 16].t().contiguous()
        total += t
        size += t.abs()
    return total, size


def within(got, a, b):
    want, size = product(a, b)
    return bool(((got.double() - want).abs() <= 1e-6 * size).all())


# ---- the products ---------------------------------------------------------------


def check_rows(m_a, u_a, m_b, experts, slots, N, K):
    """Ragged segments: skewed popularity, an expert without slots, some dropped."""
    ids = routing(slots, 1, experts, slots + N, drop=0.05, skew=0.8, busy=experts - 1)
    off, _, order, _ = plain_plan(ids, experts)
    p = fb.expert_plan(torch.from_numpy(ids).cuda(), experts)
    g = torch.Generator(device="cuda").manual_seed(K)
    x = torch.empty((slots, K), device="cuda").normal_(generator=g).abs_()
    w = torch.empty((experts * N, K), device="cuda").normal_(0.0, 0.02, generator=g)
    A, _ = fb.quantize_experts(x, p, gather=True, m=m_a, cols=False)
    out = torch.full((slots + 64, N), 7.0, device="cuda")  # (rows before and behind: whole lines for any N)
    fb.gemm_experts(A, fb.quantize(w, m=m_b), p, m_a=u_a, out=out[32:-32])
    assert bool((out[:32] == 7.0).all()) and bool((out[-32:] == 7.0).all())
    C, a = out[32:-32], bfp64(x, m_a, u_a)[torch.from_numpy(order).cuda()]
    for e in range(experts):
        if off[e + 1] > off[e]:
            r = slice(off[e], off[e + 1])
            assert within(C[r], a[r], bfp64(w[e * N:(e + 1) * N], m_b)), e
    assert off[-1] < slots and not bool(C[off[-1]:].any())


# Whole slabs of 128 of K, and rows that end inside one (exponents at any alignment).
WHOLE, RAGGED = (256, 384, 1024), (400, 1072)


@pytest.mark.parametrize("ks,ns", [(WHOLE, ODD), (RAGGED, ODD), (WHOLE, LINES)], ids=["odd", "ragged", "lines"])
@pytest.mark.parametrize("tile", [128, 0], ids=["tile128", "large"])
@pytest.mark.parametrize("m_a,u_a,m_b", FORMATS)
def test_tiled(m_a, u_a, m_b, tile, ks, ns):
    found = sizes_for(m_a, u_a, m_b, (tile, None), ks, ns)
    if tile == 0 and (u_a, m_b) in LARGE_IS_128:
        assert found is None
        return
    assert found, "no size of the grid runs on this tile"
    announce("products (%d of %d, %d) on tile %d: %d experts, %d slots, %d x %d" % (u_a, m_a, m_b, tile, *found))
    check_rows(m_a, u_a, m_b, *found)


@pytest.mark.parametrize("waves,ks", [(1, (256, 400)), (2, (1072, 1104)), (4, (2064, 2080))])
@pytest.mark.parametrize("rows", [16, 32])
@pytest.mark.parametrize("m_a,u_a,m_b", FORMATS)
def test_few_tokens(m_a, u_a, m_b, rows, waves, ks):
    found = sizes_for(m_a, u_a, m_b, (rows, waves), ks)
    if rows == 32 and u_a not in ONE_PLANE:
        assert found is None  # (32 rows of two planes do not fit the registers)
        return
    assert found, "no size of the grid runs on this kernel"
    announce("products (%d of %d, %d) on %d rows, %d waves: %d experts, %d slots, %d x %d"
             % (u_a, m_a, m_b, rows, waves, *found))
    check_rows(m_a, u_a, m_b, *found)


@pytest.mark.parametrize("m_a,u_a,m_b", [(2, 2, 8), (4, 4, 4), (6, 6, 4), (8, 8, 8)])
def test_few_tokens_many_columns(m_a, u_a, m_b):
    """Workgroups that take several groups of tiles, the last ones ragged."""
    found = (8, 32, 16387, 400)
    announce("products (%d of %d, %d) of few tokens, %d experts, %d slots, %d x %d" % (u_a, m_a, m_b, *found))
    assert rows_route(m_a, u_a, m_b, *found) == (16, 1)
    check_rows(m_a, u_a, m_b, *found)


@pytest.mark.parametrize("tile", [128, 0], ids=["tile128", "large"])
@pytest.mark.parametrize("m_a,m_b", itertools.product(WIDTHS, WIDTHS))
def test_gradients(m_a, m_b, tile):
    found = grad_sizes_for(m_a, m_b, tile)
    if tile == 0 and (m_a, m_b) in LARGE_IS_128:
        assert found is None
        return
    assert found, "no size of the grid runs on this tile"
    experts, tokens, M, N = found
    announce("gradients (%d, %d) on tile %d: %d experts, %d tokens, %d x %d" % (m_a, m_b, tile, *found))
    ids = routing(tokens, 1, experts, tokens + M, drop=0.05, skew=0.8, busy=experts - 1)
    off, koff, order, _ = plain_plan(ids, experts)
    p = fb.expert_plan(torch.from_numpy(ids).cuda(), experts)
    assert grad_route(m_a, m_b, experts, M, N, p.places) == tile
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.empty((tokens, N), device="cuda").normal_(generator=g).abs_()
    dy = torch.empty((tokens, M), device="cuda").normal_(0.0, 1e-4, generator=g)  # (in the experts' order)
    _, A = fb.quantize_experts(dy, p, m=m_a, rows=False)
    _, B = fb.quantize_experts(x, p, gather=True, m=m_b, rows=False)
    out = torch.full((experts + 2, M, N), 7.0, device="cuda")
    fb.gemm_experts_grad(A, B, p, out=out[1:-1])
    assert bool((out[0] == 7.0).all()) and bool((out[-1] == 7.0).all())
    xs = x[torch.from_numpy(order).cuda()]
    for e in range(experts):
        n = int(off[e + 1] - off[e])
        if n == 0:
            assert not bool(out[1 + e].any())
            continue
        pad = (0, 0, 0, -n % 16)
        a, b = (bfp64(torch.nn.functional.pad(t[off[e]:off[e + 1]], pad).t().contiguous(), m)
                for t, m in ((dy, m_a), (xs, m_b)))
        assert within(out[1 + e], a, b), e
    assert np.any(np.diff(koff) == 0)


@pytest.mark.parametrize("m_a,m_b", [(1, 3), (3, 1), (3, 5), (5, 7), (7, 5), (7, 7), (1, 7), (5, 1)])
@pytest.mark.parametrize("rows", [16, 128, 0])
def test_odd_widths(m_a, m_b, rows):
    found = sizes_for(m_a, m_a, m_b, (rows, None), (256, 400))
    if found is None:
        assert rows == 0 and m_a > 4 and m_b > 4  # (one tile for two planes of each)
        return
    announce("products (%d, %d) on %d rows: %d experts, %d slots, %d x %d" % (m_a, m_b, rows, *found))
    check_rows(m_a, m_a, m_b, *found)


def test_nothing_to_add():
    """K = 0: products of nothing are zeros."""
    announce("products over no values")
    ids = torch.tensor([0, 1, 1, 2, -1], device="cuda")
    p = fb.expert_plan(ids, 3)
    A, _ = fb.quantize_experts(torch.zeros((5, 0), device="cuda"), p, gather=True, cols=False)
    W = fb.quantize(torch.zeros((3 * 8, 0), device="cuda"))
    out = torch.full((5, 8), 7.0, device="cuda")
    assert not bool(fb.gemm_experts(A, W, p, out=out).any())
