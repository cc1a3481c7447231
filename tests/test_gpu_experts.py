"""The expert layer (plan, conversions in the experts' order, products of experts,
weighted sums) against plain forms in 64 bits and the oracle's conversions.

Tolerances, fixed before the first run:
  plan, conversions    equal
  products             1e-6 * sum over groups |T_G|, the library's contract for
                       every GEMM (exact group sums, FP32 sums over groups)
  weighted sum         (top + 1) 2^-24 * sum_j |g_j y_j|: one rounding for each
                       product and each sum
  gradients of it      one rounding for dy; for dgates, a lane adds ceil(N / 64) + 1
                       products and a tree of at most 8 levels adds the lanes:
                       (N / 64 + 10) 2^-24 * sum |dout y|
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import paper_2110_15456_amd as fb
from experts_util import plan as plain_plan
from experts_util import routing, token_places
from gpu_util import announce, check_tensor

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def make_plan(ids, experts, dtype=torch.int64):
    p = fb.expert_plan(torch.from_numpy(ids).to(dtype).cuda(), experts)
    return p, plain_plan(ids, experts)


# ---- the plan ---------------------------------------------------------------

PLANS = [
    # tokens, top, experts, drop, skew, busy
    (1, 1, 1, 0.0, 0.0, None),
    (1, 2, 8, 0.0, 0.0, None),
    (0, 2, 8, 0.0, 0.0, None),
    (5, 1, 3, 1.0, 0.0, None),      # everything dropped
    (63, 1, 5, 0.3, 0.0, None),
    (64, 3, 63, 0.0, 0.0, None),    # 63 experts and the tail: one chunk of 64 segments
    (129, 2, 64, 0.1, 0.0, None),   # two chunks
    (300, 2, 512, 0.0, 1.2, None),
    (2048, 2, 7, 0.1, 0.0, 1),      # one workgroup, whole; all on one expert
    (4097, 1, 9, 0.1, 1.2, None),   # two workgroups
    (9000, 6, 130, 0.2, 0.5, None),
    (1025, 1, 6, 0.1, 0.0, None),   # one workgroup, from one slot a lane to four
    (16384, 1, 8, 0.1, 0.5, None),  # the most that one workgroup takes
    (8193, 2, 8, 0.1, 0.5, None),   # and more: two launches
]


@pytest.mark.parametrize("tokens,top,experts,drop,skew,busy", PLANS)
@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_plan(tokens, top, experts, drop, skew, busy, dtype):
    top = min(top, busy or experts)
    announce("plan %d x %d of %d experts" % (tokens, top, experts))
    ids = routing(tokens, top, experts, 11, drop, skew, busy)
    p, (off, koff, order, place) = make_plan(ids, experts, dtype)
    assert np.array_equal(p.offsets.cpu().numpy(), off)
    assert np.array_equal(p.k_offsets.cpu().numpy(), koff)
    assert np.array_equal(p.order.cpu().numpy(), order)
    assert np.array_equal(p.place.cpu().numpy(), place)
    assert p.places % 128 == 0 and p.places >= koff[-1]


def test_plan_extreme_ids():
    """Ids whose low 32 bits would name an expert, and the types' limits, are dropped."""
    announce("plan with extreme ids")
    ids = np.array([[2 ** 32, 1], [-2 ** 63, 2 ** 63 - 1], [0, 2 ** 32 + 1]], dtype=np.int64)
    p, want = make_plan(ids, 4)
    assert np.array_equal(p.offsets.cpu().numpy(), want[0]) and np.array_equal(p.order.cpu().numpy(), want[2])


# ---- conversions ------------------------------------------------------------

CONVERSIONS = [
    # tokens, top, experts, drop, C
    (1, 1, 1, 0.0, 16),
    (1, 2, 8, 0.0, 48),
    (7, 2, 3, 0.3, 80),       # (C / 16 odd: a lane's two groups of a row straddle rows)
    (130, 1, 1, 0.0, 64),     # an expert of 130: two runs of 128 places
    (200, 3, 9, 0.1, 272),
    (96, 2, 70, 0.0, 128),    # more experts than one chunk of 64
]


@pytest.mark.parametrize("tokens,top,experts,drop,C", CONVERSIONS)
@pytest.mark.parametrize("m", [2, 4, 6, 8])
@pytest.mark.parametrize("mode", ["nearest", "stochastic", "truncate"])
def test_conversions(tokens, top, experts, drop, C, m, mode):
    announce("conversion %d x %d of %d experts, C = %d, m = %d, %s" % (tokens, top, experts, C, m, mode))
    ids = routing(tokens, top, experts, 5, drop)
    p, (off, koff, order, _) = make_plan(ids, experts)
    rng = np.random.Generator(np.random.PCG64(tokens + C))
    x = rng.standard_normal((tokens, C)).astype(np.float32)
    xs = np.ascontiguousarray(x[order // top])
    kept = int(off[-1])
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    xt, xst = torch.from_numpy(x).cuda(), torch.from_numpy(xs).cuda()
    wide = token_places(xs, off, koff, p.places)
    for gather, src in ((True, xt), (False, xst)):
        kw = dict(gather=gather, m=m, rounding=mode, seed_rows=21, seed_cols=22, status=st)
        both = fb.quantize_experts(src, p, **kw)
        rows = (fb.quantize_experts(src, p, cols=False, **kw)[0], None)
        cols = (None, fb.quantize_experts(src, p, rows=False, **kw)[1])
        for tr, tc in (both, rows, cols):
            if tr is not None and kept:
                check_tensor(tr, xs, 1, 16, m, mode, 21, rows=(0, kept))
            if tc is not None:
                check_tensor(tc, wide, 0, 16, m, mode, 22)
    assert int(st.item()) == 0


def test_conversion_status():
    announce("conversion of infinities")
    ids = np.array([[0, 1], [1, -1], [2, 0]])
    p, _ = make_plan(ids, 3)
    x = torch.ones((3, 32), device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    fb.quantize_experts(x, p, gather=True, status=st)
    assert int(st.item()) == 0
    x[2, 5] = float("inf")
    for kw in (dict(), dict(rows=False), dict(cols=False)):
        st.zero_()
        fb.quantize_experts(x, p, gather=True, status=st, **kw)
        assert int(st.item()) == 1


# ---- products ---------------------------------------------------------------


def values(x, m, mode="nearest", seed=0):
    """The values that x [rows, len] stands for in BFP, from the oracle, in 64 bits."""
    q, e, _ = oracle.quantize(np.ascontiguousarray(x), g=16, m=m, mode=mode, seed=seed, threads=16)
    return oracle.dequantize(q, e, 16, m).astype(np.float64).reshape(x.shape)


def drop_low(x, m, used):
    """BFP values stored at m bits, used at fewer: magnitudes without their low bits."""
    if used == m:
        return x
    v = x.reshape(-1, 16)
    q, e, _ = oracle.quantize(v.astype(np.float32), g=16, m=m)
    unit = np.ldexp(1.0, e.astype(np.int64).reshape(-1, 1) - 127 - (m - 1))
    return (np.sign(v) * (np.round(np.abs(v) / unit) // 2 ** (m - used)) * 2.0 ** (m - used) * unit).reshape(x.shape)


def bound(a, b):
    """sum over groups of |T_G| for a [M, K], b [N, K]."""
    s = np.zeros((a.shape[0], b.shape[0]))
    for k in range(0, a.shape[1], 16):
        s += np.abs(a[:, k:k + 16] @ b[:, k:k + 16].T)
    return s


PRODUCTS = [
    # tokens, top, experts, drop, skew, busy, N, K
    (1, 1, 1, 0.0, 0.0, None, 1, 16),
    (1, 2, 8, 0.0, 0.0, None, 33, 256),       # few tokens, one wave's superstep
    (16, 2, 8, 0.0, 0.0, None, 100, 2064),    # more supersteps than waves, K no multiple of 32
    (5, 1, 3, 1.0, 0.0, None, 40, 128),       # everything dropped: zeros
    (40, 2, 4, 0.2, 0.0, 2, 65, 144),         # experts without tokens
    (120, 2, 5, 0.1, 0.5, None, 130, 272),    # means of 32 to 512 slots: tiles of 128 rows
    (700, 1, 3, 0.1, 1.2, None, 260, 400),
    (1100, 2, 3, 0.05, 0.5, None, 300, 256),  # more: tiles of 256 rows
    (300, 1, 200, 0.0, 1.2, None, 16, 64),    # more experts than three chunks of 64
    (513, 1, 1, 0.0, 0.0, None, 129, 128),
]
WIDTHS = [(2, 2), (2, 4), (4, 2), (4, 4), (2, 6), (6, 2), (4, 6), (6, 4), (6, 6), (2, 8), (8, 4), (6, 8), (8, 6), (8, 8)]


@pytest.mark.parametrize("tokens,top,experts,drop,skew,busy,N,K", PRODUCTS)
def test_products(tokens, top, experts, drop, skew, busy, N, K):
    ids = routing(tokens, top, experts, 3, drop, skew, busy)
    p, (off, _, order, _) = make_plan(ids, experts)
    rng = np.random.Generator(np.random.PCG64(N + K))
    x = np.abs(rng.standard_normal((tokens, K))).astype(np.float32)
    w = (0.02 * rng.standard_normal((experts * N, K))).astype(np.float32)
    xt, wt = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    for ma, mb in WIDTHS:
        announce("products %d x %d of %d experts, %d x %d, (%d, %d)" % (tokens, top, experts, N, K, ma, mb))
        A, _ = fb.quantize_experts(xt, p, gather=True, m=ma, cols=False)
        W = fb.quantize(wt, m=mb)
        a, b = values(x, ma)[order // top], values(w, mb)
        used = [(ma, mb)] + ([(ma - (2 if ma == 6 else 4), mb)] if ma > 4 else [])
        for ua, ub in used:
            C = fb.gemm_experts(A, W, p, m_a=ua, m_b=ub).cpu().numpy().astype(np.float64)
            au = drop_low(a, ma, ua)
            for e in range(experts):
                r, be = slice(off[e], off[e + 1]), b[e * N:(e + 1) * N]
                if off[e + 1] > off[e]:
                    err = np.abs(C[r] - au[r] @ be.T)
                    assert np.all(err <= 1e-6 * bound(au[r], be) + 1e-300), (e, ua, ub, err.max())
            assert not C[off[-1]:].any()


def test_products_leave_other_columns():
    """A row stride above N, and poison around: only the N columns are written."""
    announce("products into a wider matrix")
    ids = routing(50, 2, 4, 9, 0.2)
    p, _ = make_plan(ids, 4)
    x = torch.randn((50, 64), device="cuda")
    W = fb.quantize(torch.randn((4 * 37, 64), device="cuda"))
    A, _ = fb.quantize_experts(x, p, gather=True, cols=False)
    want = fb.gemm_experts(A, W, p)
    buf = torch.full((100, 41), 7.0, device="cuda")
    lib = fb.load()
    assert lib.bfp_gemm_experts(A.mant.data_ptr(), A.exp.data_ptr(), 4, W.mant.data_ptr(), W.exp.data_ptr(), 4,
                                p.offsets.data_ptr(), 4, 100, 37, 64, 4, 4, buf.data_ptr(), 41,
                                torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(buf[:, :37], want) and bool((buf[:, 37:] == 7.0).all())


GRADS = [
    # tokens, top, experts, drop, skew, busy, M, N
    (1, 1, 1, 0.0, 0.0, None, 16, 16),
    (1, 2, 8, 0.0, 0.0, None, 48, 32),
    (5, 1, 3, 1.0, 0.0, None, 32, 64),
    (300, 2, 5, 0.1, 1.2, None, 144, 272),
    (700, 1, 2, 0.0, 0.0, 1, 32, 160),
    (600, 2, 3, 0.1, 0.5, None, 2064, 80),
]


@pytest.mark.parametrize("tokens,top,experts,drop,skew,busy,M,N", GRADS)
def test_weight_gradients(tokens, top, experts, drop, skew, busy, M, N):
    ids = routing(tokens, top, experts, 4, drop, skew, busy)
    p, (off, koff, order, _) = make_plan(ids, experts)
    rng = np.random.Generator(np.random.PCG64(M + N))
    x = np.abs(rng.standard_normal((tokens, N))).astype(np.float32)
    dy = (1e-4 * rng.laplace(size=(tokens * top, M))).astype(np.float32)
    xs = np.ascontiguousarray(x[order // top])
    xw, dw = (token_places(v, off, koff, p.places) for v in (xs, dy))
    for ma, mb in WIDTHS:
        announce("weight gradients %d x %d of %d experts, %d x %d, (%d, %d)" % (tokens, top, experts, M, N, ma, mb))
        _, A = fb.quantize_experts(torch.from_numpy(dy).cuda(), p, m=ma, rows=False)
        _, B = fb.quantize_experts(torch.from_numpy(x).cuda(), p, gather=True, m=mb, rows=False)
        G = fb.gemm_experts_grad(A, B, p).cpu().numpy().astype(np.float64)
        a, b = values(dw.T, ma), values(xw.T, mb)
        for e in range(experts):
            k = slice(koff[e], koff[e + 1])
            err = np.abs(G[e] - a[:, k] @ b[:, k].T)
            assert np.all(err <= 1e-6 * bound(a[:, k], b[:, k]) + 1e-300), (e, ma, mb, err.max())
            if koff[e] == koff[e + 1]:
                assert not G[e].any()


def test_no_tokens():
    """An empty batch: nothing to write but the weights' gradients, zeros."""
    announce("expert layer without tokens")
    p = fb.expert_plan(torch.zeros((0, 2), dtype=torch.int64, device="cuda"), 3)
    x = torch.zeros((0, 32), device="cuda")
    tr, tc = fb.quantize_experts(x, p, gather=True)
    W = fb.quantize(torch.randn((3 * 8, 32), device="cuda"))
    y = fb.gemm_experts(tr, W, p)
    assert tuple(y.shape) == (0, 8) and tuple(fb.combine_experts(y, p).shape) == (0, 8)
    _, dt = fb.quantize_experts(torch.zeros((0, 16), device="cuda"), p)
    out = torch.full((3, 16, 32), 7.0, device="cuda")
    assert not bool(fb.gemm_experts_grad(dt, tc, p, out=out).any())


def test_gradients_against_differences():
    """Of small whole numbers, which BFP at 8 bits holds exactly, so that the layer
    is linear and every sum exact: <dX, d> is the forward's change along d, and
    <dW, D> that along D."""
    announce("gradients against differences")
    T, k, E, I, O = 60, 2, 5, 64, 48
    rng = np.random.Generator(np.random.PCG64(8))
    whole = lambda *shape: torch.from_numpy(rng.integers(-3, 4, shape).astype(np.float32)).cuda()  # noqa: E731
    p, _ = make_plan(routing(T, k, E, 6, 0.2), E)
    x, w, d, D, r = whole(T, I), whole(E, O, I), whole(T, I), whole(E, O, I), whole(T, O)
    gates = whole(T, k)

    def forward(x, w, gates):
        A, _ = fb.quantize_experts(x, p, gather=True, m=8, cols=False)
        y = fb.gemm_experts(A, fb.quantize(w, m=8), p)
        return y, fb.combine_experts(y, p, gates)

    def dot(a, b):
        return float((a.double() * b.double()).sum())

    y, out = forward(x, w, gates)
    dy, dgates = fb.combine_experts_grad(r, y, p, gates)
    assert float(dy.abs().max()) < 128
    dyr, dyt = fb.quantize_experts(dy, p, m=8)
    _, xt = fb.quantize_experts(x, p, gather=True, m=8, rows=False)
    dx = fb.combine_experts(fb.gemm_experts(dyr, fb.quantize(w, group_axis=1, m=8), p), p)
    dw = fb.gemm_experts_grad(dyt, xt, p)
    base = dot(out, r)
    assert dot(forward(x + d, w, gates)[1], r) - base == dot(dx, d)
    assert dot(forward(x, w + D, gates)[1], r) - base == dot(dw, D)
    step = whole(T, k)
    assert dot(forward(x, w, gates + step)[1], r) - base == dot(dgates, step)


# ---- weighted sums ------------------------------------------------------------

COMBINES = [
    # tokens, top, experts, drop, N
    (1, 1, 1, 0.0, 1),
    (1, 2, 8, 0.0, 4096),
    (17, 3, 5, 0.3, 777),
    (3, 2, 4, 1.0, 64),       # everything dropped
    (2100, 2, 9, 0.1, 260),   # a wave for each slot
    (2100, 2, 9, 0.1, 33),
]


@pytest.mark.parametrize("tokens,top,experts,drop,N", COMBINES)
@pytest.mark.parametrize("gated", [True, False])
def test_weighted_sums(tokens, top, experts, drop, N, gated):
    announce("weighted sums %d x %d of %d experts, N = %d" % (tokens, top, experts, N))
    ids = routing(tokens, top, experts, 7, drop)
    p, (off, _, order, place) = make_plan(ids, experts)
    rng = np.random.Generator(np.random.PCG64(N))
    y = rng.standard_normal((tokens * top, N)).astype(np.float32)
    g = rng.random((tokens, top)).astype(np.float32) if gated else np.ones((tokens, top), np.float32)
    dout = rng.standard_normal((tokens, N)).astype(np.float32)
    y[off[-1]:] = np.nan  # rows of dropped choices are not read
    gt = torch.from_numpy(g).cuda() if gated else None
    yt, dt = torch.from_numpy(y).cuda(), torch.from_numpy(dout).cuda()
    out = fb.combine_experts(yt, p, gt).cpu().numpy()
    dy, dg = (t.cpu().numpy() for t in fb.combine_experts_grad(dt, yt, p, gt))
    live = (place < off[-1]).reshape(tokens, top)
    ys = np.where(live[..., None], y[place].reshape(tokens, top, N).astype(np.float64), 0.0)
    terms = np.where(live, g, 0.0).astype(np.float64)[..., None] * ys
    assert np.all(np.abs(out - terms.sum(1)) <= (top + 1) * EPS * np.abs(terms).sum(1))
    want = np.where(live[..., None], (g[..., None] * dout[:, None, :]).astype(np.float32), 0.0)
    assert np.array_equal(dy[place].reshape(tokens, top, N), want)
    prods = dout[:, None, :].astype(np.float64) * ys
    assert np.all(np.abs(dg - prods.sum(2)) <= (N / 64 + 10) * EPS * np.abs(prods).sum(2))


def test_unaligned_rows():
    """Rows that start off a 16-byte boundary take the kernels that go value by value."""
    announce("weighted sums of unaligned rows")
    p, _ = make_plan(routing(40, 2, 4, 2), 4)
    flat = torch.randn(80 * 64 + 1, device="cuda")
    y = flat[1:].view(80, 64)
    gates = torch.rand((40, 2), device="cuda")
    assert torch.equal(fb.combine_experts(y, p, gates), fb.combine_experts(y.clone(), p, gates))


def test_another_stream():
    """A plan made on one stream and used on another behind it, and the same results
    on every stream."""
    announce("expert layer on another stream")
    ids = torch.from_numpy(routing(200, 2, 6, 1)).cuda()
    x = torch.randn((200, 128), device="cuda")
    W = fb.quantize(torch.randn((6 * 96, 128), device="cuda"))
    torch.cuda.synchronize()

    def layer():
        p = fb.expert_plan(ids, 6)
        A, _ = fb.quantize_experts(x, p, gather=True, cols=False)
        return fb.combine_experts(fb.gemm_experts(A, W, p), p)

    want = layer()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = layer()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


def test_graph():
    """The layer in a graph, replayed on other routings with eager work between."""
    announce("expert layer in a graph")
    T, k, E, K, N = 300, 2, 12, 256, 200
    ids = torch.zeros((T, k), dtype=torch.int64, device="cuda")
    x = torch.zeros((T, K), device="cuda")
    W = fb.quantize(torch.randn((E * N, K), device="cuda"))
    gates = torch.rand((T, k), device="cuda")

    def layer():
        p = fb.expert_plan(ids, E)
        A, _ = fb.quantize_experts(x, p, gather=True, cols=False)
        y = fb.gemm_experts(A, W, p)
        return y, fb.combine_experts(y, p, gates), p.order

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer()
    for i in range(4):
        ids.copy_(torch.from_numpy(routing(T, k, E, 40 + i, 0.1 * i, 0.4 * i)).cuda())
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, layer()):
            assert torch.equal(a, b)


def test_bad_plans_stay_inside():
    """Offsets that are no plan (past the end, falling, negative): the products clamp
    them to the matrix; nothing outside C is written."""
    announce("products with offsets that are no plan")
    E, S, N, K = 3, 40, 32, 64
    A = fb.quantize(torch.randn((S, K), device="cuda"))
    W = fb.quantize(torch.randn((E * N, K), device="cuda"))
    buf = torch.full((3 * S, N), 7.0, device="cuda")
    lib = fb.load()
    for off in ([0, 1000, 2000, 3000], [-5, 30, 10, 2 ** 31 - 1], [40, 40, 40, 40], [30, 20, 10, 0],
                [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1]):
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        assert lib.bfp_gemm_experts(A.mant.data_ptr(), A.exp.data_ptr(), 4, W.mant.data_ptr(), W.exp.data_ptr(), 4,
                                    o.data_ptr(), E, S, N, K, 4, 4, buf[S:].data_ptr(), N,
                                    torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert bool((buf[:S] == 7.0).all()) and bool((buf[2 * S:] == 7.0).all())


def test_refusals():
    ids = torch.zeros((4, 2), dtype=torch.int64, device="cuda")
    p = fb.expert_plan(ids, 3)
    x = torch.zeros((4, 32), device="cuda")
    A, At = fb.quantize_experts(x, p, gather=True)
    W = fb.quantize(torch.zeros((3 * 8, 32), device="cuda"))
    with pytest.raises(TypeError):
        fb.expert_plan(ids.float(), 3)
    with pytest.raises(TypeError):
        fb.expert_plan(ids.cpu(), 3)
    with pytest.raises(ValueError):
        fb.expert_plan(ids[None], 3)
    with pytest.raises(ValueError):
        fb.expert_plan(ids.t(), 3)
    for n in (0, -1, 513):
        with pytest.raises(fb.BFPError):
            fb.expert_plan(ids, n)
    for bad in (dict(m=9), dict(m=0)):
        with pytest.raises(fb.BFPError):
            fb.quantize_experts(x, p, gather=True, **bad)
    for bad in (dict(gather=False), dict(gather=True, rounding="up"), dict(gather=True, rows=False, cols=False)):
        with pytest.raises(ValueError):
            fb.quantize_experts(x, p, **bad)
    with pytest.raises(ValueError):
        fb.quantize_experts(torch.zeros((4, 24), device="cuda"), p, gather=True)
    with pytest.raises(TypeError):
        fb.quantize_experts(x.double(), p, gather=True)
    with pytest.raises(ValueError):
        fb.gemm_experts(A, fb.quantize(torch.zeros((25, 32), device="cuda")), p)
    with pytest.raises(ValueError):
        fb.gemm_experts(A, fb.quantize(torch.zeros((24, 32), device="cuda"), g=32), p)
    with pytest.raises(ValueError):
        fb.gemm_experts(fb.quantize(x), W, p)
    with pytest.raises(fb.BFPError):
        fb.gemm_experts(A, W, p, m_a=3)
    with pytest.raises(ValueError):
        fb.gemm_experts_grad(A, A, p)
    with pytest.raises(ValueError):
        fb.combine_experts(x, p)
    y = torch.zeros((8, 32), device="cuda")
    with pytest.raises(ValueError):
        fb.combine_experts(y, p, torch.zeros((4, 3), device="cuda"))
    with pytest.raises(ValueError):
        fb.combine_experts_grad(y, y, p)
    with pytest.raises(fb.BFPError):
        fb.combine_experts_grad(x, y, p, out=y)
