"""What the orthogonalised update's two FP16 planes hold of rows far weaker than the
rest, row by row.

Tolerance, fixed before the first run.  An entry of X is held to 2^-23 of itself or
2^-40, an entry of S to 2^-40 and of P to 2^-39 (their scales are 2^15, 2^15 and
2^14, FP16's smallest step is 2^-24).  In a row of X' = P X that leaves, besides what
FP32 would leave (four times its error and 2^-22 of the row, as for whole
matrices), 2^-40 sqrt(k) from X and, with nearly orthonormal rows of at most 1.21,
sqrt(n) times P's error, 2^-39 and |b| + 2 c |S| = 10.7 times that of S: less than 16
2^-40 sqrt(n).  Each of the steps grows it by at most a = 3.4445, so that the sum over
the steps is below 1.5 a^steps."""
from __future__ import annotations

import pytest
import torch

import paper_2110_15456_amd as fb
from gpu_util import announce

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315


def plain(u, steps, eps=1e-7):
    x = u / (u.norm() + eps)
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = A * x + (B * s + C * (s @ s)) @ x
    return x


@pytest.mark.parametrize("n,k", [(64, 576), (120, 200), (300, 1100), (1024, 1024), (1000, 4100)])
@pytest.mark.parametrize("weak", [1.0, 1e-3, 1e-6, 1e-9])
@pytest.mark.parametrize("steps", [5, 12])
def test_weak_rows(n, k, weak, steps):
    announce("orthogonalize %d x %d, half of the rows at %g, %d steps" % (n, k, weak, steps))
    u = torch.randn((n, k), generator=torch.Generator(device="cuda").manual_seed(n + k), device="cuda")
    u[1::2] *= weak
    want = plain(u.double(), steps)
    low = (plain(u, steps).double() - want).norm(dim=1)
    err = (fb.orthogonalize(u, steps=steps).double() - want).norm(dim=1)
    floor = 1.5 * A ** steps * 2.0 ** -40 * (k ** 0.5 + 16 * n ** 0.5)
    # (a row's FP32 error by chance below its neighbours': the largest of its kind)
    for rows in (slice(0, None, 2), slice(1, None, 2)):
        assert bool((err[rows] <= 4 * low[rows].max() + 2.0 ** -22 * want[rows].norm(dim=1) + floor).all())


@pytest.mark.parametrize("n,k", [(64, 576), (1000, 4100)])
def test_weak_columns(n, k):
    """The transpose's weak columns are the same rows."""
    announce("orthogonalize %d x %d, weak columns" % (n, k))
    u = torch.randn((n, k), generator=torch.Generator(device="cuda").manual_seed(n), device="cuda")
    u[1::2] *= 1e-4
    assert torch.equal(fb.orthogonalize(u.t().contiguous()).t(), fb.orthogonalize(u))


# Fixed before the first run: no less accurate than the formula in FP32 on the same
# input, in the mean over eight draws; a quarter more for the draws themselves.
@pytest.mark.parametrize("n,k", [(16, 16), (48, 48), (64, 576), (32, 1000), (96, 300), (128, 128), (128, 1152), (160, 160),
                                 (256, 512), (512, 512)])
@pytest.mark.parametrize("strong", [0, 8], ids=["noise", "strong"])
def test_no_less_accurate_than_fp32(n, k, strong):
    announce("orthogonalize %d x %d against FP32, %d strong directions" % (n, k, strong))
    ours = low = 0.0
    for seed in range(8):
        g = torch.Generator(device="cuda").manual_seed(100 + seed)
        u = 1e-4 * torch.randn((n, k), generator=g, device="cuda")
        if strong:
            u += 1e-2 / k ** 0.5 * (torch.randn((n, strong), generator=g, device="cuda") @
                                    torch.randn((strong, k), generator=g, device="cuda"))
        want = plain(u.double(), 5)
        size = float(want.norm())
        ours += float((fb.orthogonalize(u).double() - want).norm()) / size / 8
        low += float((plain(u, 5).double() - want).norm()) / size / 8
    assert ours <= 1.25 * low, (ours, low)
