"""The operators of a linear layer's training step in 8-bit floating point behind a
norm, each in its plain form and as the framework's calls, over the range of sizes
and types that such layers have.

Kinds of case
  norm       a residual's addition and the root-mean-square norm of the sum, with the
             output converted to 8 bits (e4m3 or e5m2, a power-of-two scale for each
             128 values of a row) or left in FP32
  norm_grad  its gradients: to the sum (with the residual path's own) and to the weights
  linear     activations converted to 8 bits and multiplied with weights held in 8 bits,
             the result in BF16
  backward   a linear layer's backward pass: the output's gradient converted along both
             axes, the input along its tokens, and the two products, in BF16
  clip       the norm over all gradients of a model, and the gradients scaled down to a
             largest norm, into the buffers that the update reads

The residual stream is FP32; what passes between it and the products is BF16 or FP32
("t" of a case).

Inputs are drawn from the seed: normal activations with a few strong channels, N(0,
0.02) weights, Laplace(0, 1e-4) gradients with 1% of the entries scaled by 100.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
# of a format: its type, the exponent of its largest power of two
FORMATS = {"e4m3": (torch.float8_e4m3fn, 8), "e5m2": (torch.float8_e5m2, 15)}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the smallest call: one token of a 4096-wide model, where launches and the host show
        dict(name="norm_one_token", kind="norm", rows=1, d=4096, residual=True, to="e4m3", t="bf16"),
        # a middling batch of an odd width, without a residual, FP32 out (a head's input)
        dict(name="norm_ragged", kind="norm", rows=1531, d=777, residual=False, to="fp32", t="fp32"),
        # a full batch in front of an 8-bit product
        dict(name="norm_full", kind="norm", rows=8192, d=4096, residual=True, to="e4m3", t="bf16"),
        # a short batch's backward pass at an odd width
        dict(name="norm_grad_ragged", kind="norm_grad", rows=700, d=1155, residual=False, t="fp32"),
        # a full batch's
        dict(name="norm_grad_full", kind="norm_grad", rows=8192, d=4096, residual=True, t="bf16"),
        # decoding: 16 tokens against the FFN up-projection, bound by the weights' bytes
        dict(name="linear_decode", kind="linear", tokens=16, d_in=4096, d_out=16384, fmt="e4m3", t="bf16"),
        # a middling batch of odd sizes, in the format of wide range
        dict(name="linear_ragged", kind="linear", tokens=1531, d_in=1050, d_out=777, fmt="e5m2", t="fp32"),
        # a full batch of tokens through the FFN up-projection
        dict(name="linear_full", kind="linear", tokens=8192, d_in=4096, d_out=16384, fmt="e4m3", t="bf16"),
        # a full batch's backward pass through a projection as wide as the model
        dict(name="backward_full", kind="backward", tokens=8192, d_in=4096, d_out=4096, fmt="e4m3", t="bf16"),
        # the gradients of one small layer
        dict(name="clip_layer", kind="clip", tensors=8, total=1 << 20, ratio=3.0, t="fp32"),
        # of a model of many tensors of odd sizes
        dict(name="clip_many", kind="clip", tensors=150, total=40_000_001, ratio=3.0, t="bf16"),
        # of a large model's share
        dict(name="clip_full", kind="clip", tensors=24, total=400_000_000, ratio=3.0, t="fp32"),
    ]


def _log(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "linear", "linear", "backward", "clip"])
    if kind in ("norm", "norm_grad"):
        rows, d = _log(rng, 1, 16384), _log(rng, 16, 16384)
        while rows * d > 8192 * 4096:
            rows = rows * 3 // 4
        case = dict(kind=kind, rows=rows, d=d, residual=rng.random() < 0.7, t=rng.choice(["fp32", "bf16"]))
        if kind == "norm" and not case["residual"]:
            case["t"] = "fp32"  # (the stream itself)
        return dict(case, to=rng.choice(["e4m3", "e4m3", "e5m2", "fp32"])) if kind == "norm" else case
    if kind == "clip":
        tensors = _log(rng, 1, 300)
        return dict(kind=kind, tensors=tensors, total=max(tensors, _log(rng, 10_000, 200_000_000)),
                    ratio=rng.choice([0.5, 3.0]), t=rng.choice(["fp32", "bf16"]))
    tokens, d_in, d_out = _log(rng, 1, 8192), _log(rng, 64, 16384), _log(rng, 64, 16384)
    while tokens * d_in * d_out > 8192 * 4096 * 4096 or tokens * (d_in + d_out) > 1 << 28:
        if d_in > d_out:
            d_in = d_in * 3 // 4
        else:
            d_out = d_out * 3 // 4
    if rng.random() < 0.5:
        d_in, d_out = -(-d_in // 16) * 16, -(-d_out // 16) * 16
    return dict(kind=kind, tokens=tokens, d_in=d_in, d_out=d_out, fmt=rng.choice(["e4m3", "e4m3", "e5m2"]),
                t=rng.choice(["fp32", "bf16"]))


# ---- inputs -------------------------------------------------------------


def _values(what, shape, gen):
    x = torch.empty(shape, dtype=torch.float32, device="cuda")
    if what == "activations":
        x.normal_(generator=gen)
        strong = torch.empty(shape[-1], device="cuda").uniform_(0.0, 1.0, generator=gen) < 0.01
        return x * torch.where(strong, 20.0, 1.0)
    if what == "weights":
        return x.normal_(0.0, 0.02, generator=gen)
    x.exponential_(1e4, generator=gen)
    u = torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(-1.0, 1.0, generator=gen)
    x = torch.where(u.abs() < 0.01, 100.0 * x, x)
    return torch.where(u < 0, -x, x)


def _lengths(case, seed):
    """The tensors' sizes: `total` values over `tensors` tensors, a few of them most of it."""
    g = torch.Generator().manual_seed(seed)
    n, total = case["tensors"], case["total"]
    share = torch.exp(2.0 * torch.randn(n, generator=g, dtype=torch.float64))
    sizes = [1 + int(v) for v in (share / share.sum() * (total - n)).tolist()]
    sizes[0] += total - sum(sizes)
    return sizes


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, t = case["kind"], TYPES[case["t"]]
    if kind == "clip":
        flat = _values("grads", (case["total"],), gen).to(t)
        norm = math.sqrt(case["total"] * 2e-8 * (1.0 + 0.01 * 9999.0))  # (expected)
        return dict(flat=flat, sizes=_lengths(case, seed), max_norm=norm / case["ratio"])
    if kind in ("norm", "norm_grad"):
        shape = (case["rows"], case["d"])
        v = dict(x=_values("activations", shape, gen), w=1.0 + 5.0 * _values("weights", shape[1:], gen))
        if case["residual"]:
            v["residual"] = _values("activations", shape, gen) if kind == "norm" else _values("grads", shape, gen)
        if kind == "norm_grad":
            return dict(v, dy=_values("grads", shape, gen).to(t))
        return dict(v, x=v["x"].to(t))
    T, I, O = case["tokens"], case["d_in"], case["d_out"]
    v = dict(x=_values("activations", (T, I), gen).to(t), w=_values("weights", (O, I), gen))
    if kind == "backward":
        v["dy"] = _values("grads", (T, O), gen).to(t)
    return v


def prepare(case, seed):
    """What a training or serving program has in hand: the inputs, the layer's weights
    in 8 bits (the plain forms hold the values that they stand for), what the forward
    pass left for the backward one, and the list of a model's gradients with the
    buffers that their scaled values go to (one bucket, as an exchange has it)."""
    v = _inputs(case, seed)
    kind, s = case["kind"], dict(case=case, **v)
    if own:
        import paper_2110_15456_amd as fb
    if kind == "clip":
        s["grads"] = [g.clone() for g in torch.split(s.pop("flat"), v["sizes"])]
        s["bucket"] = torch.empty(case["total"], dtype=TYPES[case["t"]], device="cuda")
        if own:
            s["list"] = fb.tensor_list(s["grads"], out=torch.split(s["bucket"], v["sizes"]))
    elif kind == "norm_grad":
        s["r"] = _inverse_rms(v["x"]).float()
    elif kind == "linear":
        s["w"] = fb.quantize_fp8(v["w"], fmt=case["fmt"]) if own else _rounded(v["w"], case["fmt"])
    elif kind == "backward":  # the weights along their outputs
        s["w"] = (fb.quantize_fp8(v["w"], axis=0, fmt=case["fmt"]) if own
                  else _rounded(v["w"].t().contiguous(), case["fmt"]))
    return s


# ---- the plain forms ----------------------------------------------------


def _to_fp8(x, fmt):
    """Codes [rows, d] and scale bytes [rows, blocks] of x: of each 128 values of a row
    (the last block of a row may be shorter) the least power of two by which the
    largest value is within the format."""
    kind, top = FORMATS[fmt]
    rows, d = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -d % 128)).reshape(rows, -1, 128)
    bits = v.abs().amax(dim=2, keepdim=True).view(torch.int32)
    scale = ((bits >> 23) + ((bits & 0x7FFFFF) > 0x600000) - top).clamp(min=0)  # (above 1.75 * 2^e: the next one)
    codes = (v * ((254 - scale) << 23).view(torch.float32)).to(kind)
    return codes.reshape(rows, -1)[:, :d], scale[:, :, 0].to(torch.uint8)


def _rounded(x, fmt):
    """The values that x has in 8 bits."""
    codes, scale = _to_fp8(x, fmt)
    back = (scale.to(torch.int32) << 23).view(torch.float32)
    return codes.float() * torch.repeat_interleave(back, 128, dim=1)[:, :x.shape[1]]


def _inverse_rms(h):
    return torch.rsqrt(h.double().square().mean(dim=1) + EPS)


def _norm(s):
    h = s["x"] + s["residual"] if "residual" in s else s["x"]
    y = (h.double() * _inverse_rms(h)[:, None] * s["w"].double()).float()
    out = dict(h=h) if "residual" in s else {}
    if s["case"]["to"] == "fp32":
        return dict(out, y=y)
    codes, scale = _to_fp8(y, s["case"]["to"])
    return dict(out, y=codes, scale=scale)


def _norm_grad(s):
    h, r, d, dy = s["x"], s["r"][:, None], s["case"]["d"], s["dy"].float()
    u = s["w"] * dy
    dx = r * u - h * (r * r * r * ((u * h).sum(dim=1, keepdim=True) / d))
    dx = dx + s["residual"] if "residual" in s else dx
    return dict(dx=dx, dw=(dy * (h * r)).sum(dim=0))


def _backward(s):
    fmt = s["case"]["fmt"]
    dx = torch.mm(_rounded(s["dy"], fmt), s["w"].t())
    dw = torch.mm(_rounded(s["dy"].t().contiguous(), fmt), _rounded(s["x"].t().contiguous(), fmt).t())
    return dict(dx=dx.bfloat16(), dw=dw.bfloat16())


def _clip(s):
    flat = torch.cat(s["grads"])
    norm = flat.double().square().sum().sqrt()
    return dict(grads=(flat.double() * (s["max_norm"] / norm).clamp(max=1.0)).to(flat.dtype), norm=norm.reshape(1))


# ---- one pass -----------------------------------------------------------


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if not own:
        if kind == "linear":
            return dict(y=torch.mm(_rounded(s["x"], case["fmt"]), s["w"].t()).bfloat16())
        return {"norm": _norm, "norm_grad": _norm_grad, "backward": _backward, "clip": _clip}[kind](s)
    import paper_2110_15456_amd as fb
    if kind == "norm":
        to = None if case["to"] == "fp32" else case["to"]
        y, h, _ = fb.rms_norm(s["x"], s["w"], residual=s.get("residual"), eps=EPS, to=to)
        out = dict(h=h) if case["residual"] else {}
        return dict(out, y=y) if to is None else dict(out, y=y.codes, scale=y.exp)
    if kind == "norm_grad":
        dx, dw = fb.rms_norm_grad(s["dy"], s["x"], s["r"], s["w"], dresidual=s.get("residual"))
        return dict(dx=dx, dw=dw)
    if kind == "linear":
        return dict(y=fb.gemm_fp8(fb.quantize_fp8(s["x"], fmt=case["fmt"]), s["w"], dtype=torch.bfloat16))
    if kind == "backward":
        dy, dyt = fb.quantize_fp8_dual(s["dy"], fmt=case["fmt"])
        xt = fb.quantize_fp8(s["x"], axis=0, fmt=case["fmt"])
        return dict(dx=fb.gemm_fp8(dy, s["w"], dtype=torch.bfloat16), dw=fb.gemm_fp8(dyt, xt, dtype=torch.bfloat16))
    norm = fb.clip_gradients(s["list"], s["max_norm"])
    return dict(grads=s["bucket"], norm=norm)


# ---- what a pass cannot do without --------------------------------------


def work(case):
    kind, t = case["kind"], 4.0 if case["t"] == "fp32" else 2.0
    if kind == "clip":  # the gradients in, the scaled ones out
        return dict(bytes=2.0 * t * case["total"], flops=3.0 * case["total"])
    if kind in ("norm", "norm_grad"):
        n = float(case["rows"]) * case["d"]
        if kind == "norm_grad":  # dy and h (and the residual path's gradient) in, dx out
            return dict(bytes=n * (t + 8.0 + 4.0 * case["residual"]) + 8.0 * case["d"] + 4.0 * case["rows"],
                        flops=10.0 * n)
        # x (and the residual) in, the norm's output (and the sum) out
        return dict(bytes=n * (t + 8.0 * case["residual"] + (4.0 if case["to"] == "fp32" else 1.0 + 1.0 / 128.0))
                    + 4.0 * case["d"], flops=5.0 * n)
    T, I, O = case["tokens"], case["d_in"], case["d_out"]
    stored = 1.0 + 1.0 / 128.0
    if kind == "linear":  # x and the weights in, y out
        return dict(bytes=t * T * I + stored * I * O + 2.0 * T * O, flops=2.0 * T * I * O)
    # x, dy and the weights in, dx and dw out
    return dict(bytes=(t + 2.0) * T * I + t * T * O + stored * I * O + 2.0 * I * O, flops=4.0 * T * I * O)


# ---- the same in 64 bits ------------------------------------------------


def _two(e):
    """2^e in 64 bits, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _fp8_64(x, fmt):
    """The values that x has in 8 bits and the scales' bytes, from the definition: of
    each block the scale is the least power of two with no value above the format's
    largest, and a value goes to the nearest multiple of its place, ties to even."""
    bits, least, most = {"e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0)}[fmt]
    rows, d = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -d % 128)).reshape(rows, -1, 128)
    top = v.abs().amax(dim=2, keepdim=True)
    m, e = torch.frexp(top / most)  # top / most = m 2^e with m in [1/2, 1)
    power = torch.where(top > 0, torch.where(m == 0.5, e - 1, e), torch.full_like(e, -127)).clamp(min=-127)
    v = v * _two(-power)
    place = torch.frexp(v)[1].sub(1).clamp(min=least) - bits
    v = torch.round(v * _two(-place)) * _two(place + power)
    return v.reshape(rows, -1)[:, :d], (power[:, :, 0] + 127).to(torch.uint8)


def exact(case, seed):
    v = _inputs(case, seed)
    kind = case["kind"]
    if kind == "clip":
        g = v["flat"].double()
        norm = torch.linalg.vector_norm(g)
        return dict(grads=g * (v["max_norm"] / norm) if norm > v["max_norm"] else g, norm=norm.reshape(1))
    if kind == "norm":
        h = v["x"]
        if case["residual"]:
            h = (h.double() + v["residual"].double()).float()
        out = dict(h=h.double()) if case["residual"] else {}
        h = h.double()
        y = h / torch.sqrt((h * h).sum(dim=1, keepdim=True) / case["d"] + EPS) * v["w"].double()
        if case["to"] == "fp32":
            return dict(out, y=y)
        values, scale = _fp8_64(y.float(), case["to"])  # (of the norm's FP32 value)
        codes = values * torch.repeat_interleave(_two(127 - scale.to(torch.int32)), 128, dim=1)[:, :case["d"]]
        return dict(out, y=codes, scale=None)
    if kind == "norm_grad":
        h, dy, d = v["x"].double(), v["dy"].double(), case["d"]
        r = 1.0 / torch.sqrt((h * h).sum(dim=1, keepdim=True) / d + EPS)
        n = h * r
        u = dy * v["w"].double()
        dx = r * (u - n * (u * n).mean(dim=1, keepdim=True))
        return dict(dx=dx + v["residual"].double() if case["residual"] else dx, dw=(dy * n).sum(dim=0))
    x, w, fmt = v["x"], v["w"], case["fmt"]
    if kind == "linear":
        return dict(y=_fp8_64(x, fmt)[0] @ _fp8_64(w, fmt)[0].t())
    dy = v["dy"]
    dx = _fp8_64(dy, fmt)[0] @ _fp8_64(w.t().contiguous(), fmt)[0].t()
    return dict(dx=dx, dw=_fp8_64(dy.t().contiguous(), fmt)[0] @ _fp8_64(x.t().contiguous(), fmt)[0].t())
