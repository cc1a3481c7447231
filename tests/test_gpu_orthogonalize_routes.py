"""The orthogonalised update on every tile, number of stages and splitting of its
products that the prices choose, against the formula in 64 bits.

Sizes are looked for: the cheapest of a grid that the library says it takes a
variant for, so that other prices lead to other sizes and not to variants that no
test runs.  Tolerance, fixed before the first run, as in test_gpu_orthogonalize.py:
four times the error of the formula in FP32 on the same input, and 2^-22 of the
norm."""
from __future__ import annotations

import ctypes
import functools

import pytest
import torch

import paper_2110_15456_amd as fb
from gpu_util import announce

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315

BATCHES = (1, 2, 3, 5, 7, 12, 14, 20, 37, 40, 62)
SIZES = (40, 70, 134, 200, 356, 407, 504, 700, 882, 977, 1015, 1300, 1610, 2050, 2219, 2500, 2980, 3050, 3110, 3780,
         4500, 6300)
SIDES = [(r, c) for r in SIZES for c in SIZES]


def kind(whole, parts, tiles):
    return "whole" if parts == 1 or whole == tiles else "parts" if whole == 0 else "mixed"


@functools.lru_cache(maxsize=None)
def variants(batch, rows, cols):
    """What an update of this size runs: (product, tile, stages, how)."""
    tile, stages, parts = (ctypes.c_int * 3)(), (ctypes.c_int * 3)(), (ctypes.c_int * 2)()
    whole = (ctypes.c_int64 * 2)()
    assert fb.load().bfp_orthogonalize_route(batch, rows, cols, tile, stages, parts, whole) == 0
    n, out = min(rows, cols), {("write", tile[2], stages[2], "transposed" if rows > cols else "plain")}
    for i, name in enumerate(("gram", "square")):
        t = -(-n // tile[i])
        how = kind(whole[i], parts[i], batch * t * (t + 1) // 2)
        if n > 128:
            out.add((name, tile[i], stages[i], how))
        elif i == 0:  # (the symmetric products are one kernel, which adds the parts)
            out.add(("small", -(-n // 32), stages[i], "parts" if parts[i] > 1 else "whole"))
    return out


@functools.lru_cache(maxsize=None)
def cheapest(variant):
    best = None
    for batch in BATCHES:
        for rows, cols in SIDES:
            cost = batch * rows * cols * min(rows, cols)
            if variant[0] == "square" and max(rows, cols) < 1.25 * min(rows, cols):
                continue  # (steps in pairs have all of the symmetric products)
            if batch * rows * cols <= 1 << 27 and (best is None or cost < best[0]) and variant in variants(batch, rows,
                                                                                                           cols):
                best = (cost, batch, rows, cols)
    return best and best[1:]


def reached():
    seen = set()
    for batch in BATCHES:
        for rows, cols in SIDES:
            if batch * rows * cols <= 1 << 27:
                seen |= variants(batch, rows, cols)
    return seen


VARIANTS = sorted([("gram", t, 2, how) for t in (64, 128, 256) for how in ("whole", "parts", "mixed")] +
                  [("square", t, 2, how) for t in (64, 128, 256) for how in ("whole", "parts", "mixed")] +
                  [(name, 64, 4, how) for name in ("gram", "square") for how in ("whole", "parts")] +
                  [("small", t, 4, how) for t in (2, 3) for how in ("whole", "parts")] + [("small", 2, 2, "parts")] +
                  [("write", t, 2, how) for t in (64, 128, 256) for how in ("plain", "transposed")] +
                  [("write", 64, 4, how) for how in ("plain", "transposed")])


def plain(u, steps=5, eps=1e-7):
    """The iteration on one matrix with no more rows than columns, in its type."""
    x = u / (u.norm() + eps)
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = A * x + (B * s + C * (s @ s)) @ x
    return x


@pytest.mark.parametrize("variant", VARIANTS, ids=lambda v: "-".join(map(str, v)))
def test_variant(variant):
    size = cheapest(variant)
    assert size, "no size of the grid takes it"
    announce("orthogonalize %d x %d x %d, %s" % (*size, variant))
    batch, rows, cols = size
    r = min(3, rows, cols)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    u = 1e-4 * torch.randn(size, generator=g, device="cuda")
    for i in range(batch):  # (every other matrix: strong directions over the noise)
        if i % 2 == 0:
            u[i] += 1e-2 * (torch.randn((rows, r), generator=g, device="cuda") @
                            torch.randn((r, cols), generator=g, device="cuda"))
    buf = torch.full((batch * rows * cols + 512,), 7.0, device="cuda")
    out = buf[256:-256].view(size)
    fb.orthogonalize(u, out=out)
    assert bool((buf[:256] == 7.0).all()) and bool((buf[-256:] == 7.0).all())
    for i in range(batch):
        flip = rows > cols
        v, got = (t.t().contiguous() if flip else t for t in (u[i], out[i]))
        want = plain(v.double())
        low = float((plain(v).double() - want).norm())
        err = float((got.double() - want).norm())
        assert err <= 4 * low + 2.0 ** -22 * float(want.norm()), (i, err, low)


def test_every_variant_is_listed():
    """Nothing on the grid runs a variant that is not tested (the small matrices'
    kernels of other edges are test_gpu_orthogonalize.py's)."""
    assert {v for v in reached() if v[0] != "small"} <= set(VARIANTS)
