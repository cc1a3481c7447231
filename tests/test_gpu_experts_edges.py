"""The expert layer's calls at the edges of what they take."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2110_15456_amd as fb
from gpu_util import announce

pytestmark = pytest.mark.gpu


def test_weighted_sum_over_its_input():
    """One choice a token: out has y's shape, but the rows change places."""
    announce("weighted sum over its input is refused")
    p = fb.expert_plan(torch.tensor([2, 0, 1, 0], device="cuda"), 3)
    y = torch.randn((4, 32), device="cuda")
    with pytest.raises(fb.BFPError):
        fb.combine_experts(y, p, out=y)
    with pytest.raises(fb.BFPError):
        fb.combine_experts_grad(y, y.clone(), p, out=y)


# Beyond 2^20 slots a workgroup of the plan takes several rounds.
@pytest.mark.parametrize("slots,experts,dtype", [(1 << 20, 8, torch.int32), ((1 << 20) + 1, 8, torch.int64),
                                                 (2500001, 130, torch.int32), (4194305, 512, torch.int64)])
def test_plan_of_many_slots(slots, experts, dtype):
    announce("plan of %d slots, %d experts" % (slots, experts))
    rng = np.random.Generator(np.random.PCG64(slots))
    ids = np.minimum(rng.geometric(2.0 / experts, slots) - 1, experts)  # skewed; the id past the end: dropped
    p = fb.expert_plan(torch.from_numpy(ids).to(dtype).cuda(), experts)
    counts = np.bincount(ids, minlength=experts + 1)[:experts]
    order = np.argsort(ids, kind="stable")
    assert np.array_equal(p.offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(counts)]))
    assert np.array_equal(p.k_offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(-(-counts // 128) * 128)]))
    assert np.array_equal(p.order.cpu().numpy(), order)
    place = np.empty_like(order)
    place[order] = np.arange(slots)
    assert np.array_equal(p.place.cpu().numpy(), place)


# An odd number of groups in a row (a lane's two straddle rows), and rows that end with
# a lane, a wave and a workgroup.
@pytest.mark.parametrize("C", [16, 48, 1024, 8192])
@pytest.mark.parametrize("m", [2, 4, 6, 8])
def test_status_of_dropped_slots(C, m):
    """What a dropped slot's row holds sets no status, whichever outputs are asked for;
    what the row before it holds does."""
    announce("status of dropped slots, C = %d, m = %d" % (C, m))
    ids = torch.tensor([[1, -1], [0, 5], [-1, -1], [0, 1], [-1, 0]], device="cuda")  # 5 of 10 kept; token 2 has none
    p = fb.expert_plan(ids, 2)
    kept = 5
    assert int(p.offsets[-1]) == kept
    asked = [dict(), dict(cols=False), dict(rows=False)]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def status(x, **kw):
        st.zero_()
        fb.quantize_experts(x, p, m=m, status=st, **kw)
        return int(st.item())

    x = torch.ones((10, C), device="cuda")
    for at in (0, C - 1):
        for value in (float("nan"), float("inf")):
            poison = x.clone()
            poison[kept:, at] = value
            assert [status(poison, **kw) for kw in asked] == [0, 0, 0], (at, value)
            poison[kept - 1, at] = value
            assert [status(poison, **kw) for kw in asked] == [1, 1, 1], (at, value)
            tokens = x[:5].clone()
            tokens[2, at] = value
            assert [status(tokens, gather=True, **kw) for kw in asked] == [0, 0, 0], (at, value)
            tokens[4, at] = value
            assert [status(tokens, gather=True, **kw) for kw in asked] == [1, 1, 1], (at, value)


@pytest.mark.parametrize("gather", [True, False])
def test_status_leaves_the_bytes(gather):
    """Asking for the status changes no byte of what is written."""
    announce("conversions with and without a status")
    ids = torch.tensor([[1, -1], [0, 5], [-1, -1], [0, 1], [-1, 0]], device="cuda")
    p = fb.expert_plan(ids, 2)
    x = torch.randn((5 if gather else 10, 272), device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    for m in (2, 4, 6, 8):
        a, _ = fb.quantize_experts(x, p, gather=gather, m=m, cols=False)
        b, _ = fb.quantize_experts(x, p, gather=gather, m=m, cols=False, status=st)
        assert torch.equal(a.mant, b.mant) and torch.equal(a.exp, b.exp)


def test_gates_in_another_order():
    """[top, tokens] holds as many gates as [tokens, top], in another order."""
    announce("gates of a wrong shape are refused")
    p = fb.expert_plan(torch.tensor([[0, 1], [1, 2], [2, 0]], device="cuda"), 3)
    y, dout = torch.randn((6, 16), device="cuda"), torch.randn((3, 16), device="cuda")
    gates = torch.rand((3, 2), device="cuda")
    want = fb.combine_experts(y, p, gates)
    assert torch.equal(fb.combine_experts(y, p, gates.reshape(-1)), want)  # the slots in order
    for bad in (gates.t().contiguous(), gates.reshape(6, 1), gates.reshape(1, 6), gates[:2].contiguous()):
        with pytest.raises(ValueError):
            fb.combine_experts(y, p, bad)
        with pytest.raises(ValueError):
            fb.combine_experts_grad(dout, y, p, bad)
    one = fb.expert_plan(torch.tensor([0, 2, 1, 1, 0, 2], device="cuda"), 3)  # one choice each
    g = gates.reshape(6)
    assert torch.equal(fb.combine_experts(y, one, g), fb.combine_experts(y, one, g[:, None].contiguous()))


def losing_terms(n):
    """n values near 1 of which every sum in order loses nearly half a unit in its last
    place, so that n FP32 sums in a row are off by about 0.35 n 2^-24 of the result."""
    out, s = np.empty(n, np.float32), np.float32(0)
    for i in range(n):
        out[i] = np.float32(1.0 + 0.49 * np.spacing(s)) if s >= 2 else np.float32(1)
        s = np.float32(s + out[i])
    return out


# Slots that take four waves each, and one: the columns from one of a lane's to its next.
@pytest.mark.parametrize("tokens,top,N,stride", [(1, 1, 262144, 1024), (3, 2, 262144, 1024), (4099, 1, 4096, 256),
                                                 (2100, 2, 4095, 64)])
def test_gate_gradients_of_long_rows(tokens, top, N, stride):
    """dgates at most 5 2^-24 of the terms' absolute sum off, whatever N is: four
    products and their sums in FP32, 2^-24 each; the rounding of the result; and sums
    in 64 bits, N 2^-53.  The terms lose all they can in one FP32 sum a lane."""
    announce("gate gradients, %d x %d, N = %d" % (tokens, top, N))
    c = np.arange(N)
    v = 4 if N % 4 == 0 else 1
    row = losing_terms(N // stride * v + v)[c // stride * v + c % v]
    rng = np.random.Generator(np.random.PCG64(N))
    ids = np.argsort(rng.random((tokens, 5)), axis=1)[:, :top]
    p = fb.expert_plan(torch.from_numpy(ids).cuda(), 5)
    scale = np.ldexp(1.0, rng.integers(-3, 4, tokens * top)).astype(np.float32)  # (exact; tells the slots apart)
    y = torch.from_numpy(row).cuda()[None] * torch.from_numpy(scale).cuda()[:, None]
    _, dg = fb.combine_experts_grad(torch.ones((tokens, N), device="cuda"), y, p)
    want = row.astype(np.float64).sum() * scale[p.place.cpu().numpy()].reshape(tokens, top)
    err = np.abs(dg.cpu().numpy() - want) / want
    assert np.all(err <= 5 * 2.0 ** -24 + N * 2.0 ** -53), err.max() * 2 ** 24


@pytest.mark.parametrize("N", [48, 40])
def test_update_of_every_experts_weights(N):
    """The update of a batch of matrices, taken to the weights and their two groupings
    as the binding describes, is each expert's own (N a multiple of 16 or not: the
    grouping along N needs one)."""
    announce("weights of experts updated, N = %d" % N)
    E, K = 3, 64
    w, grad = torch.randn((E, N, K), device="cuda"), torch.randn((E, N, K), device="cuda")
    step, momentum = fb.orthogonal_update(grad, torch.zeros_like(grad))
    new = w.clone().add_(step, alpha=-0.5)
    along_k = fb.quantize(new)
    along_n = fb.quantize(new, group_axis=1) if N % 16 == 0 else None
    for e in range(E):
        one, m_one = fb.orthogonal_update(grad[e].contiguous(), torch.zeros_like(grad[e]))
        assert torch.equal(m_one, momentum[e])
        assert float((one - step[e]).norm()) <= 1e-4 * float(one.norm())  # (another batch: other parts of the sums)
        if along_n is None:
            continue
        _, rows, cols = fb.weight_update(w[e].contiguous(), step[e].contiguous(), -0.5)
        r, c = slice(e * N, (e + 1) * N), slice(e * K, (e + 1) * K)
        assert torch.equal(rows.exp, along_k.exp[r]) and torch.equal(cols.exp, along_n.exp[c])
        assert torch.equal(fb.dequantize(rows), fb.dequantize(along_k)[r])
        assert torch.equal(fb.dequantize(cols), fb.dequantize(along_n)[c])
