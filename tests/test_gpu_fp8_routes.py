"""Every kernel that the prices of 8-bit products know, in every format, with exact
integer data: sizes are looked up by the route, so that all of them run whatever the prices
are, at odd numbers of rows, columns and slabs, with K in parts and whole."""
from __future__ import annotations

import ctypes
import functools
import random

import numpy as np
import pytest
import torch

import paper_2110_15456_amd as fb
from paper_2110_15456_amd import _lib
from tests import fp8_util as F

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KERNELS = [(64, 64, 0), (128, 128, 0), (256, 256, 0), (16, 16, 4), (16, 64, 2), (32, 32, 2)]


def route(M, N, K, room=1 << 40):
    out = [ctypes.c_int(0) for _ in range(4)]
    _lib.check(_lib.load().bfp_gemm_fp8_route(M, N, K, room, *[ctypes.byref(o) for o in out]), "route")
    return tuple(o.value for o in out)


@functools.lru_cache(maxsize=None)
def sizes(kernel, split):
    """Up to three ragged sizes that the kernel takes, of few slabs and of many."""
    rng = random.Random(3)
    found = []
    for _ in range(100000):
        M, N = (int(2 ** rng.uniform(11 if kernel[0] == 256 and not split else 0, 13)) for _ in range(2))
        K = int(2 ** rng.uniform(0, 14 if split else 12))
        if M * N > 2 ** 25 or M * N * K > 2 ** 35 or M % 16 == 0 or N % 16 == 0:
            continue
        r = route(M, N, K)
        if r[:3] == kernel and (r[3] > 1) == split and (len(found) != 1 or (-(-K // 128) - -(-found[0][2] // 128)) % 2):
            found.append((M, N, K))
            if len(found) == 3:
                break
    return found


@pytest.mark.parametrize("fmt_a,fmt_b", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("kernel,split", [(k, s) for k in KERNELS for s in ((False, True) if k[2] == 0 else (False,))])
def test_kernel(kernel, split, fmt_a, fmt_b):
    found = sizes(kernel, split)
    assert found, "no size takes this kernel"
    for M, N, K in found:
        print(kernel, split, fmt_a, fmt_b, M, N, K, route(M, N, K), flush=True)
        gen = torch.Generator(device=DEV).manual_seed(K)

        def draw(rows, fmt):
            t = fb.FP8Tensor.empty(rows, K, fmt, DEV)
            v = torch.randint(-7, 8, (rows, t.data.shape[1]), generator=gen, device=DEV)
            v[:, K:] = 0
            table = torch.from_numpy(np.searchsorted(F.table(fmt), np.arange(8.0)).astype(np.uint8)).to(DEV)
            t.data.view(torch.uint8).copy_(table[v.abs()] | (v < 0).to(torch.uint8) * 0x80)
            e = torch.randint(126, 129, tuple(t.scales.shape), generator=gen, device=DEV)
            t.scales.copy_(e)
            unit = torch.repeat_interleave(torch.exp2(e.double() - 127).round(decimals=1), 128, dim=1)[:, :v.shape[1]]
            return t, v.double() * unit

        (A, a), (B, b) = draw(M, fmt_a), draw(N, fmt_b)
        C = (a @ b.t().contiguous())
        guard = torch.full((M + 2, N), 5.0, device=DEV)
        fb.gemm_fp8(A, B, out=guard[1:M + 1])
        assert torch.equal(guard[1:M + 1].double(), C)
        assert bool((guard[0] == 5).all()) and bool((guard[M + 1] == 5).all())
        assert torch.equal(fb.gemm_fp8(A, B, dtype=torch.bfloat16), C.float().bfloat16())
        # rows that are whole lines leave past the caches
        wide = torch.empty((M, (N + 63) // 64 * 64), device=DEV)
        fb.gemm_fp8(A, B, out=wide[:, :N])
        assert torch.equal(wide[:, :N].double(), C)
