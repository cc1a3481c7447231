"""The operators of an expert layer (a mixture of experts' feed-forward layer in
BFP) and of its weight update, each in its plain form and as the framework's
calls, over the range of sizes and types that such layers have.

Kinds of case
  linear    the forward of an expert layer: tokens sent to experts of their own,
            converted to BFP in the experts' order and multiplied with their
            expert's weights (held in BFP); ragged numbers of tokens, experts
            without any, choices that a capacity limit dropped
  backward  its backward pass: both groupings of dY, the gradient of every
            token (summed over its experts) and of every expert's weights
  combine   the weighted sum of each token's expert outputs, and its gradients
            to the outputs and to the weights
  update    a step of momentum whose result is orthogonalised (five steps of the
            quintic Newton-Schulz iteration), as the Muon optimiser takes it

Inputs are drawn from the seed: half-normal activations, N(0, 0.02) weights,
Laplace(0, 1e-4) gradients with 1% of the entries scaled by 100 (a weight's
gradient has a few strong directions besides).  The experts of a token are
drawn without replacement, from a uniform or a skewed popularity.
"""
from __future__ import annotations

import math

import torch

own = False

BETA, EPS, STEPS = 0.95, 1e-7, 5
NS = (3.4445, -4.7750, 2.0315)  # the quintic iteration's coefficients


def listed():
    return [
        # the smallest call: one token through a 256-wide layer, where launches and the host show
        dict(name="linear_one_token", kind="linear", tokens=1, top=2, experts=8, d_in=256, d_out=256, m_x=4, m_w=4,
             skew=0.0, drop=0.0),
        # decoding: 16 tokens against the FFN up-projection of 8 experts, bound by the weights' bytes
        dict(name="linear_decode", kind="linear", tokens=16, top=2, experts=8, d_in=4096, d_out=16384, m_x=4, m_w=4,
             skew=0.0, drop=0.0),
        # a middling batch on many small experts: odd widths, mixed types, skewed popularity, dropped choices
        dict(name="linear_ragged", kind="linear", tokens=1531, top=4, experts=48, d_in=1056, d_out=777, m_x=4, m_w=6,
             skew=1.2, drop=0.1),
        # a full batch of tokens through the FFN up-projection of 8 experts
        dict(name="linear_full", kind="linear", tokens=8192, top=2, experts=8, d_in=4096, d_out=16384, m_x=4, m_w=4,
             skew=0.5, drop=0.0),
        # backward through small ragged experts, at the schedule's last width
        dict(name="backward_ragged", kind="backward", tokens=700, top=2, experts=16, d_in=576, d_out=1152, m=6,
             skew=1.2, drop=0.1),
        # backward of a full batch through 8 experts as wide as the model, at the schedule's middle width
        dict(name="backward_full", kind="backward", tokens=8192, top=2, experts=8, d_in=4096, d_out=4096, m=4,
             skew=0.5, drop=0.0),
        # a few tokens' outputs summed, and the gradients
        dict(name="combine_few", kind="combine", tokens=16, top=2, experts=8, d=4096, drop=0.0),
        # a full batch's, with some choices dropped
        dict(name="combine_full", kind="combine", tokens=8192, top=4, experts=48, d=4096, drop=0.1),
        # a small convolution's weights: 64 x 576, bound by the chain of launches
        dict(name="update_conv2", kind="update", batch=1, rows=64, cols=576),
        # the experts of a small layer in one call: odd sizes, more rows than columns
        dict(name="update_experts", kind="update", batch=16, rows=1152, cols=777),
        # the output projection: square
        dict(name="update_out_proj", kind="update", batch=1, rows=4096, cols=4096),
        # the FFN up-projection: the largest matrix
        dict(name="update_ffn_up", kind="update", batch=1, rows=16384, cols=4096),
    ]


def _log(rng, lo, hi, multiple=1):
    """A size spread over the logarithm of [lo, hi], a multiple of `multiple`."""
    v = max(multiple, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / multiple)) * multiple)
    return v + multiple if v == 3 << 10 else v


def draw(rng):
    kind = rng.choice(["linear", "linear", "backward", "combine", "update"])
    if kind == "update":
        batch, rows, cols = _log(rng, 1, 32), _log(rng, 16, 16384), _log(rng, 16, 16384)
        while batch * rows * cols > 1 << 26 or batch * rows * cols * min(rows, cols) > 4096 * 4096 * 16384:
            batch, rows, cols = (batch + 1) // 2, max(16, rows * 3 // 4), max(16, cols * 3 // 4)
        return dict(kind=kind, batch=batch, rows=rows, cols=cols)
    experts = _log(rng, 1, 128)
    tokens, top = _log(rng, 1, 8192), min(experts, rng.choice([1, 2, 2, 4, 6]))
    drop = rng.choice([0.0, 0.0, 0.1, 0.3])
    if kind == "combine":
        return dict(kind=kind, tokens=tokens, top=top, experts=experts, d=_log(rng, 16, 8192), drop=drop)
    skew = rng.choice([0.0, 0.5, 1.2])
    d_in, d_out = _log(rng, 64, 16384, 16), _log(rng, 64, 16384, 16)
    most = 8 * 4096 * (16384 if kind == "linear" else 4096)
    while experts * d_in * d_out > most or tokens * top * d_in * d_out > 2048 * most or tokens * top * (
            d_in + d_out) > 1 << 28:
        if d_in > d_out:
            d_in = max(64, d_in * 3 // 64 * 16)
        else:
            d_out = max(64, d_out * 3 // 64 * 16)
    case = dict(kind=kind, tokens=tokens, top=top, experts=experts, d_in=d_in, d_out=d_out)
    if kind == "linear":
        case.update(d_out=d_out - rng.choice([0, 0, 7]), m_x=rng.choice([2, 4, 4, 6, 8]), m_w=rng.choice([2, 4, 4, 6, 8]))
    else:
        case.update(m=rng.choice([2, 4, 6]))
    return dict(case, skew=skew, drop=drop)


# ---- inputs -------------------------------------------------------------


def _values(what, shape, gen):
    x = torch.empty(shape, dtype=torch.float32, device="cuda")
    if what == "half_normal":
        return x.normal_(generator=gen).abs_()
    if what == "weights":
        return x.normal_(0.0, 0.02, generator=gen)
    x.exponential_(1e4, generator=gen)
    u = torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(-1.0, 1.0, generator=gen)
    x = torch.where(u.abs() < 0.01, 100.0 * x, x)
    return torch.where(u < 0, -x, x)


def _weight_grads(batch, rows, cols, gen):
    """Gradients of weights: Laplace entries and, ten times as strong, eight directions."""
    r = min(8, rows, cols)
    a = torch.empty((batch, rows, r), dtype=torch.float32, device="cuda").normal_(generator=gen)
    b = torch.empty((batch, r, cols), dtype=torch.float32, device="cuda").normal_(generator=gen)
    return _values("grads", (batch, rows, cols), gen) + (1e-2 / math.sqrt(max(rows, cols))) * torch.matmul(a, b)


def _routing(case, seed):
    """The experts of every token [tokens, top], -1 for a choice that was dropped
    (made on the host, so that the plain forms need no read-back of the counts)."""
    g = torch.Generator().manual_seed(seed)
    T, k, E = case["tokens"], case["top"], case["experts"]
    popularity = -case.get("skew", 0.0) * torch.log1p(torch.randperm(E, generator=g).float())
    noise = -torch.log(-torch.log(torch.rand((T, E), generator=g).clamp(1e-9, 1 - 1e-7)))
    ids = torch.topk(popularity + noise, k, dim=1).indices
    return torch.where(torch.rand((T, k), generator=g) < case["drop"], torch.full_like(ids, -1), ids)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    if kind == "update":
        shape = (case["batch"], case["rows"], case["cols"])
        return dict(grad=_weight_grads(*shape, gen), momentum=3.0 * _weight_grads(*shape, gen))
    ids = _routing(case, seed)
    v = dict(ids=ids.cuda(), counts=torch.bincount(ids[ids >= 0], minlength=case["experts"]).tolist())
    if kind == "combine":
        S = case["tokens"] * case["top"]
        v["y"] = torch.empty((S, case["d"]), dtype=torch.float32, device="cuda").normal_(generator=gen)
        v["gates"] = torch.softmax(torch.empty((case["tokens"], case["top"]), device="cuda").normal_(generator=gen), 1)
        v["dout"] = _values("grads", (case["tokens"], case["d"]), gen)
        return v
    T, I, O, E = case["tokens"], case["d_in"], case["d_out"], case["experts"]
    v.update(x=_values("half_normal", (T, I), gen), w=_values("weights", (E, O, I), gen))
    if kind == "backward":
        v["dy"] = _values("grads", (T * case["top"], O), gen)
    return v


def prepare(case, seed):
    """What a training or serving program has in hand: the inputs, the layer's
    weights in BFP and, after the forward pass, the plan of its routing.  The
    plain forms hold the values that the BFP weights stand for."""
    v = _inputs(case, seed)
    kind, s = case["kind"], dict(case=case, **v)
    if kind == "update":
        return s
    if own:
        import paper_2110_15456_amd as fb
        if kind != "linear":
            s["plan"] = fb.expert_plan(v["ids"], case["experts"])
    elif kind != "linear":
        s["order"], s["place"] = _order(v["ids"])
    w = s.pop("w", None)
    if kind == "linear":  # [experts, d_out, d_in] in groups along d_in
        s["w"] = fb.quantize(w, m=case["m_w"]) if own else _bfp(w, case["m_w"])
    elif kind == "backward":  # [experts, d_in, d_out] in groups along d_out
        s["w"] = fb.quantize(w, group_axis=1, m=case["m"]) if own else _bfp(w.transpose(1, 2).contiguous(), case["m"])
    return s


# ---- the plain forms ----------------------------------------------------


def _bfp(x, m):
    """The values of x in BFP with groups of 16 along the last axis and m-bit
    magnitudes, rounded to nearest (half up in magnitude, saturating)."""
    v = x.reshape(-1, 16)
    e = (v.abs().amax(dim=1, keepdim=True).view(torch.int32) >> 23).clamp(min=m + 16)  # (biased; 0 for zeros)
    up = ((254 + m - e) << 23).view(torch.float32)  # 2^(m - (e - 127)): twice the magnitude in units of the last place
    q = torch.floor(0.5 * (torch.floor(v.abs() * up) + 1.0)).clamp(max=2.0 ** m - 1.0)
    return (torch.copysign(q, v) * ((e - (m - 1)) << 23).view(torch.float32)).reshape(x.shape)


def _order(ids):
    """The slots (token, choice) in the order of their experts, dropped ones last,
    and every slot's place in that order."""
    flat = ids.reshape(-1)
    order = torch.sort(torch.where(flat < 0, torch.full_like(flat, 1 << 30), flat), stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    return order, place


def _ends(counts):
    ends = [0]
    for n in counts:
        ends.append(ends[-1] + n)
    return ends


def _segments(x, w, counts):
    """x's rows (in the experts' order) times their expert's w^T; zeros for those
    without an expert.  (One product for each expert that has tokens, with the
    counts known on the host: the quickest form of elementary products.)"""
    ends = _ends(counts)
    y = x.new_zeros((x.shape[0], w.shape[1]))
    for e, n in enumerate(counts):
        if n:
            torch.mm(x[ends[e]:ends[e + 1]], w[e].t(), out=y[ends[e]:ends[e + 1]])
    return y


def _token_groups(x, m, counts):
    """BFP values of x [slots, d] with groups of 16 consecutive tokens of an expert
    (an expert's last group filled with zeros), and where each expert's begin."""
    starts = _ends([(n + 15) // 16 * 16 for n in counts])
    kept = sum(counts)
    shift = torch.repeat_interleave(
        torch.tensor([a - b for a, b in zip(starts[:-1], _ends(counts)[:-1])], device=x.device),
        torch.tensor(counts, device=x.device), output_size=kept)
    p = x.new_zeros((starts[-1], x.shape[1]))
    p[torch.arange(kept, device=x.device) + shift] = x[:kept]
    return _bfp(p.t().contiguous(), m), starts


def _linear(s):
    case = s["case"]
    order, _ = _order(s["ids"])
    x = _bfp(s["x"], case["m_x"])[order // case["top"]]
    return dict(y=_segments(x, s["w"], s["counts"]), order=order.to(torch.int32))


def _backward(s):
    case, counts = s["case"], s["counts"]
    dx = _segments(_bfp(s["dy"], case["m"]), s["w"], counts)
    dx = dx[s["place"]].reshape(case["tokens"], case["top"], -1).sum(dim=1)
    xt, starts = _token_groups(s["x"][s["order"] // case["top"]], case["m"], counts)
    dyt, _ = _token_groups(s["dy"], case["m"], counts)
    dw = torch.empty((case["experts"], case["d_out"], case["d_in"]), device=dx.device)
    for e in range(case["experts"]):
        torch.mm(dyt[:, starts[e]:starts[e + 1]], xt[:, starts[e]:starts[e + 1]].t(), out=dw[e])
    return dict(dx=dx, dw=dw)


def _combine(s):
    case = s["case"]
    T, k, d = case["tokens"], case["top"], case["d"]
    gates = torch.where(s["ids"] < 0, torch.zeros_like(s["gates"]), s["gates"])
    y = s["y"][s["place"]].reshape(T, k, d)
    out = (gates[:, :, None] * y).sum(dim=1)
    dgates = torch.where(s["ids"] < 0, torch.zeros_like(gates), (s["dout"][:, None, :] * y).sum(dim=2))
    dy = (gates.reshape(-1)[s["order"]])[:, None] * s["dout"][s["order"] // k]
    return dict(out=out, dy=dy, dgates=dgates)


def _update(s):
    a, b, c = NS
    m = BETA * s["momentum"] + s["grad"]
    x = s["grad"] + BETA * m
    x = x / (x.square().sum(dim=(1, 2), keepdim=True).sqrt() + EPS)
    wide = x.shape[1] <= x.shape[2]
    x = x if wide else x.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        g = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * g + c * torch.matmul(g, g), x)
    return dict(update=x if wide else x.transpose(1, 2).contiguous(), momentum=m)


# ---- one pass -----------------------------------------------------------


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if not own:
        return {"linear": _linear, "backward": _backward, "combine": _combine, "update": _update}[kind](s)
    import paper_2110_15456_amd as fb
    if kind == "linear":
        plan = fb.expert_plan(s["ids"], case["experts"])
        x, _ = fb.quantize_experts(s["x"], plan, gather=True, m=case["m_x"], cols=False)
        return dict(y=fb.gemm_experts(x, s["w"], plan), order=plan.order)
    if kind == "backward":
        plan, m = s["plan"], case["m"]
        _, xt = fb.quantize_experts(s["x"], plan, gather=True, m=m, rows=False)
        dy, dyt = fb.quantize_experts(s["dy"], plan, m=m)
        dx = fb.combine_experts(fb.gemm_experts(dy, s["w"], plan), plan)
        return dict(dx=dx, dw=fb.gemm_experts_grad(dyt, xt, plan))
    if kind == "combine":
        out = fb.combine_experts(s["y"], s["plan"], s["gates"])
        dy, dgates = fb.combine_experts_grad(s["dout"], s["y"], s["plan"], s["gates"])
        return dict(out=out, dy=dy, dgates=dgates)
    update, momentum = fb.orthogonal_update(s["grad"], s["momentum"], beta=BETA, steps=STEPS, eps=EPS)
    return dict(update=update, momentum=momentum)


# ---- what a pass cannot do without --------------------------------------


def _stored(n, m):
    """Bytes of n values in BFP with groups of 16 and m-bit magnitudes."""
    return n * ({2: 4, 4: 6, 6: 10, 8: 12}[m] / 8.0 + 1.0 / 16.0)


def work(case):
    kind = case["kind"]
    if kind == "update":
        b, n, k = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # the gradient and the momentum in, the update and the new momentum out; in each step the halves of
        # two symmetric products (x x^T and its square) and one full one
        return dict(bytes=16.0 * b * n * k, flops=STEPS * b * (n * (n + 1.0) * (k + n) + 2.0 * n * n * k))
    T, k, E = case["tokens"], case["top"], case["experts"]
    S = T * k
    if kind == "combine":
        # the experts' outputs and the gradient in, the sum and the outputs' gradient out
        return dict(bytes=4.0 * case["d"] * (2 * S + 2 * T) + 20.0 * S, flops=5.0 * S * case["d"])
    I, O = case["d_in"], case["d_out"]
    kept = S * (1.0 - case["drop"])
    busy = min(E, E * (1.0 - (1.0 - min(1.0, k / E)) ** T) if case.get("skew", 0.0) == 0.0 else kept)
    if kind == "linear":
        # x and the weights of the experts that have tokens in, y out
        return dict(bytes=4.0 * T * I + _stored(busy * I * O, case["m_w"]) + 4.0 * S * O + 12.0 * S,
                    flops=2.0 * kept * I * O)
    # x, dy and the busy experts' weights in, dx and every expert's dw out
    return dict(bytes=4.0 * T * I + 4.0 * S * O + _stored(busy * I * O, case["m"]) + 4.0 * T * I + 4.0 * E * I * O,
                flops=4.0 * kept * I * O)


# ---- the same in 64 bits ------------------------------------------------


def _bfp64(x, m):
    """The BFP values (groups of 16 along the last axis) from the definition: the
    exponent of the group's largest value, magnitudes in units of its last place
    with half a unit added and the fraction dropped, at most 2^m - 1."""
    v = x.double().reshape(-1, 16)
    top = v.abs().amax(dim=1, keepdim=True)
    unit = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - m), torch.ones_like(top))
    return (torch.sign(v) * torch.clamp(torch.floor(v.abs() / unit + 0.5), max=2 ** m - 1) * unit).reshape(x.shape)


def exact(case, seed):
    v = _inputs(case, seed)
    kind = case["kind"]
    if kind == "update":
        a, b, c = NS
        m = v["momentum"].double() * BETA + v["grad"].double()
        out = []
        for x in v["grad"].double() + BETA * m:
            x = x / (torch.linalg.norm(x) + EPS)
            x = x.t().contiguous() if x.shape[0] > x.shape[1] else x
            for _ in range(STEPS):
                g = x @ x.t()
                x = a * x + (b * g + c * (g @ g)) @ x
            out.append(x.t() if case["rows"] > case["cols"] else x)
        return dict(update=torch.stack(out), momentum=m)
    ids, T, k = v["ids"].cpu(), case["tokens"], case["top"]
    flat = ids.reshape(-1).tolist()
    slots = [[] for _ in range(case["experts"] + 1)]  # of each expert, then the dropped ones
    for i, e in enumerate(flat):
        slots[e].append(i)  # (-1: the last list)
    order = torch.tensor([i for part in slots for i in part])
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k)
    order, place, kept = order.cuda(), place.cuda(), sum(v["counts"])
    token = order // k
    if kind == "combine":
        y, dout = v["y"].double(), v["dout"].double()
        out, dy = torch.zeros_like(dout), torch.zeros_like(y)
        dgates = torch.zeros(T * k, dtype=torch.float64, device="cuda")
        g = v["gates"].double().reshape(-1)[order[:kept]]
        out.index_add_(0, token[:kept], g[:, None] * y[:kept])
        dy[:kept] = g[:, None] * dout[token[:kept]]
        dgates[order[:kept]] = (y[:kept] * dout[token[:kept]]).sum(dim=1)
        return dict(out=out, dy=dy, dgates=dgates.reshape(T, k))
    I, O, E = case["d_in"], case["d_out"], case["experts"]
    at = 0
    if kind == "linear":
        x = _bfp64(v["x"], case["m_x"])
        y = torch.zeros((T * k, O), dtype=torch.float64, device="cuda")
        for e, n in enumerate(v["counts"]):
            if n:
                y[at:at + n] = x[token[at:at + n]] @ _bfp64(v["w"][e], case["m_w"]).t()
            at += n
        return dict(y=y, order=None)
    m = case["m"]
    dx = torch.zeros((T, I), dtype=torch.float64, device="cuda")
    dw = torch.zeros((E, O, I), dtype=torch.float64, device="cuda")
    for e, n in enumerate(v["counts"]):
        if not n:
            continue
        rows = slice(at, at + n)
        dy = v["dy"][rows]
        dx.index_add_(0, token[rows], _bfp64(dy, m) @ _bfp64(v["w"][e].t().contiguous(), m).t())
        fill = (0, 0, 0, -n % 16)
        dyt = _bfp64(torch.nn.functional.pad(dy, fill).t().contiguous(), m)
        xt = _bfp64(torch.nn.functional.pad(v["x"][token[rows]], fill).t().contiguous(), m)
        dw[e] = dyt @ xt.t()
        at += n
    return dict(dx=dx, dw=dw)
