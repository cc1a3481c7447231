"""What a layer has around its products: 8-bit floating-point blocks and their products,
the root-mean-square norm in front of one, and the clipping of a model's gradients
(bindings of include/fastbfp.h; argument checks and allocations, as in the package)."""
from __future__ import annotations

import ctypes
import functools
import math

import torch

from . import ROUNDING, BFPTensor, _need_cuda, _stream
from ._lib import check, load

# Of a format: the ABI's number and torch's type.
FP8_FORMATS = {"e4m3": (0, torch.float8_e4m3fn), "e5m2": (1, torch.float8_e5m2)}


TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _type(t, name):
    """The ABI's number of the type of a CUDA tensor, FP32 or BF16."""
    _need_cuda(t, name)
    if t.dtype not in TYPES:
        raise TypeError("%s must have dtype torch.float32 or torch.bfloat16, got %s" % (name, t.dtype))
    return TYPES[t.dtype]


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _call(name, dev, *args):
    """The library's ``name`` on dev's current stream.  dev is the current device for the
    call: the default stream's handle names the current device's."""
    f = getattr(load(), name)
    if _current_device() == dev.index:
        check(f(*args, _stream(dev)), name)
    else:
        with torch.cuda.device(dev):
            check(f(*args, _stream(dev)), name)


def _status(status, dev):
    """The address of a status word, or None."""
    if status is None:
        return None
    _need_cuda(status, "status")
    if status.dtype not in (torch.int32, torch.uint32) or status.numel() != 1:
        raise TypeError("status must be one int32 or uint32 value")
    _on(dev, status=status)
    return status.data_ptr()


def _format(fmt):
    if fmt not in FP8_FORMATS:
        raise ValueError("fmt must be one of %s" % sorted(FP8_FORMATS))
    return FP8_FORMATS[fmt]


def _on(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError("%s must be on %s" % (name, device))


def _f32(t, name, shape, dev):
    """t is a contiguous FP32 tensor of that shape on dev."""
    if isinstance(t, torch.Tensor) and t.dtype is torch.float32 and t.shape == shape and t.device == dev and t.is_contiguous():
        return
    _need_cuda(t, name, torch.float32)
    if t.shape != shape:
        raise ValueError("%s must be %s" % (name, list(shape)))
    _on(dev, **{name: t})


def _same_start(a, b):
    """Whether a is a tensor that begins where b does (others that share memory are refused
    by the library)."""
    return isinstance(a, torch.Tensor) and a.data_ptr() == b.data_ptr()


# ---- 8-bit blocks -------------------------------------------------------


class FP8Tensor:
    """A rows x len tensor of 8-bit codes with a power-of-two scale for each 128 values
    of a row (see include/fastbfp.h).

    data: float8 [rows, 128 * blocks], zeros behind a row's last value;
    scales: uint8 [rows, blocks rounded up to a multiple of 4], zeros behind the last.
    """
    __slots__ = ("rows", "len", "fmt", "device", "_data", "_scales", "_bytes", "_ptrs")

    def __init__(self, data: torch.Tensor, scales: torch.Tensor, rows: int, length: int, fmt: str):
        for name, t, dtype, pitch in (("data", data, _format(fmt)[1], _pitches(length)[0]),
                                      ("scales", scales, torch.uint8, _pitches(length)[1])):
            if t.dtype != dtype:
                raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
            if tuple(t.shape) != (rows, pitch) or not t.is_contiguous():
                raise ValueError("%s must be [%d, %d], contiguous" % (name, rows, pitch))
        if scales.device != data.device:
            raise ValueError("scales must be on %s" % data.device)
        self.rows, self.len, self.fmt, self.device = rows, length, fmt, data.device
        self._data, self._scales, self._bytes = data, scales, None
        # what the library takes: the codes' and scales' addresses, and the format
        self._ptrs = data.data_ptr(), scales.data_ptr(), _format(fmt)[0]

    @property
    def data(self) -> torch.Tensor:
        if self._data is None:
            pitch = _pitches(self.len)[0]
            self._data = self._bytes[:self.rows * pitch].view(self.rows, pitch).view(_format(self.fmt)[1])
        return self._data

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            pitch, ep = _pitches(self.len)
            self._scales = self._bytes[self.rows * pitch:].view(self.rows, ep)
        return self._scales

    @property
    def codes(self) -> torch.Tensor:
        """float8 [rows, len]: the values in units of their block's scale."""
        return self.data if self.data.shape[1] == self.len else self.data[:, :self.len]

    @property
    def exp(self) -> torch.Tensor:
        """uint8 [rows, blocks]: the scales are 2^(exp - 127)."""
        blocks = (self.len + 127) // 128
        return self.scales if self.scales.shape[1] == blocks else self.scales[:, :blocks]

    @staticmethod
    def empty(rows: int, length: int, fmt: str, device) -> "FP8Tensor":
        pitch, ep = _pitches(length)
        code, dtype = _format(fmt)
        t = FP8Tensor.__new__(FP8Tensor)
        t.rows, t.len, t.fmt = rows, length, fmt
        t._data, t._bytes = torch.empty(rows, pitch, dtype=dtype, device=device), None
        t._scales = torch.empty(rows, ep, dtype=torch.uint8, device=device)
        t.device, t._ptrs = t._data.device, (t._data.data_ptr(), t._scales.data_ptr(), code)
        return t

    @staticmethod
    def _one_buffer(rows, length, fmt, device) -> "FP8Tensor":
        """As empty, both arrays in one allocation and views of them made when asked for:
        for an operand that goes straight into a product."""
        pitch, ep = _pitches(length)
        t = FP8Tensor.__new__(FP8Tensor)
        t.rows, t.len, t.fmt, t.device = rows, length, fmt, device
        t._data = t._scales = None
        t._bytes = torch.empty(rows * (pitch + ep), dtype=torch.uint8, device=device)
        p = t._bytes.data_ptr()
        t._ptrs = p, p + rows * pitch, _format(fmt)[0]
        return t


def _pitches(length):
    """Bytes from one row's codes, and scales, to the next one's."""
    blocks = (length + 127) // 128
    return 128 * blocks, (blocks + 3) // 4 * 4


def _fp8_out(out, rows, length, fmt, device, make=FP8Tensor._one_buffer):
    if out is None:
        return make(rows, length, fmt, device)
    if (out.rows, out.len, out.fmt) != (rows, length, fmt):
        raise ValueError("out has the wrong shape or format")
    if out.device != device:
        raise ValueError("out must be on %s" % device)
    return out


def quantize_fp8(x: torch.Tensor, axis: int = -1, fmt: str = "e4m3", status: torch.Tensor | None = None,
                 out: FP8Tensor | None = None) -> FP8Tensor:
    """FP32 or BF16 -> 8-bit blocks ("e4m3" or "e5m2") along the last axis (the leading axes are
    the rows), or along axis 0 of a 2-D tensor, written transposed: a [R, C] tensor
    becomes a [C, R] one, K-contiguous for the product.  Any sizes.  ``status``: as
    quantize's."""
    code, _ = _format(fmt)
    xt = _type(x, "x")
    shape = x.shape
    nd = len(shape)
    if nd < 1 or not -nd <= axis < nd:
        raise ValueError("axis must be one of x's")
    along = axis == -1 or axis == nd - 1
    C = shape[-1]
    R = shape[0] if nd == 2 else math.prod(shape[:-1])
    if not along and nd != 2:
        raise ValueError("axis must be the last one, or 0 of a 2-D tensor")
    t = _fp8_out(out, R if along else C, C if along else R, fmt, x.device)
    codes, scales, _ = t._ptrs
    _call("bfp_quantize_fp8", x.device, x.data_ptr(), xt, R, C, 1 if along else 0, code, codes, scales,
          _status(status, x.device))
    return t


def quantize_fp8_dual(x: torch.Tensor, fmt: str = "e4m3", status: torch.Tensor | None = None,
                      out_rows: FP8Tensor | None = None, out_cols: FP8Tensor | None = None):
    """Both conversions of a 2-D tensor from one read: ``(quantize_fp8(x),
    quantize_fp8(x, axis=0))``."""
    code, _ = _format(fmt)
    xt = _type(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be 2-D")
    R, C = x.shape
    tr, tc = _fp8_out(out_rows, R, C, fmt, x.device), _fp8_out(out_cols, C, R, fmt, x.device)
    _call("bfp_quantize_fp8_dual", x.device, x.data_ptr(), xt, R, C, code, *tr._ptrs[:2], *tc._ptrs[:2],
          _status(status, x.device))
    return tr, tc


def dequantize_fp8(t: FP8Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """8-bit blocks -> FP32 [rows, len]."""
    y = out if out is not None else torch.empty((t.rows, t.len), dtype=torch.float32, device=t.device)
    _need_cuda(y, "out", torch.float32)  # (and so t, whose device it shares)
    _f32(y, "out", (t.rows, t.len), t.device)
    _call("bfp_dequantize_fp8", t.device, *t._ptrs[:2], t.rows, t.len, t._ptrs[2], y.data_ptr())
    return y


@functools.lru_cache(maxsize=4096)
def _gemm_fp8_ws(M, N, K):
    """Workspace bytes of bfp_gemm_fp8 (a function of the sizes alone)."""
    nb = ctypes.c_size_t(0)
    check(load().bfp_gemm_fp8_ws_size(M, N, K, ctypes.byref(nb)), "bfp_gemm_fp8_ws_size")
    return nb.value


def gemm_fp8_ws_size(A: FP8Tensor, B: FP8Tensor) -> int:
    """Workspace bytes with which gemm_fp8 may sum K in parts (0 for most products)."""
    return _gemm_fp8_ws(A.rows, B.rows, A.len)


def gemm_fp8(A: FP8Tensor, B: FP8Tensor, dtype: torch.dtype | None = None, out: torch.Tensor | None = None,
             workspace=True) -> torch.Tensor:
    """C = A . B^T [A.rows, B.rows] for 8-bit A [M, K] and B [N, K], in either format each.
    ``dtype``: torch.float32 (or out's) or torch.bfloat16; the matrix instruction's
    alignment of the products costs about 2^-14 of their size at random (see
    include/fastbfp.h), so FP32 saves BF16's rounding but is no FP32 sum.
    ``out``: rows may be apart (a slice of columns).  ``workspace``: True
    allocates what gemm_fp8_ws_size asks for (the product runs whole where the card has
    no room); a uint8 tensor of at least that size takes its place, and calls that share
    it must not overlap; False runs the product whole."""
    if A.len != B.len:
        raise ValueError("A and B must share K (A: %d, B: %d)" % (A.len, B.len))
    dev = A.device
    if dev.type != "cuda":
        raise TypeError("A and B must be on a CUDA (HIP) device")
    if B.device != dev:
        raise ValueError("B must be on %s" % dev)
    M, N, K = A.rows, B.rows, A.len
    if out is None:
        C, ldc = torch.empty(M, N, dtype=torch.float32 if dtype is None else dtype, device=dev), N
    else:
        C = out
        if not isinstance(C, torch.Tensor) or not C.is_cuda:
            raise TypeError("out must be a CUDA (HIP) tensor")
        if dtype is not None and C.dtype != dtype:
            raise TypeError("out must have dtype %s, got %s" % (dtype, C.dtype))
        if tuple(C.shape) != (M, N):
            raise ValueError("out must be [%d, %d]" % (M, N))
        if (N > 1 and C.stride(1) != 1) or (M > 1 and C.stride(0) < N):
            raise ValueError("out's rows must be contiguous and apart")
        _on(dev, out=C)
        ldc = C.stride(0) if M > 1 else N
    if C.dtype not in TYPES:
        raise TypeError("dtype must be torch.float32 or torch.bfloat16, got %s" % C.dtype)
    need, ws = 0, None
    if workspace is not False:
        need = _gemm_fp8_ws(M, N, K)
        if need and isinstance(workspace, torch.Tensor):
            _need_cuda(workspace, "workspace", torch.uint8)
            _on(dev, workspace=workspace)
            if workspace.numel() < need:
                raise ValueError("workspace needs %d bytes" % need)
            ws = workspace
        elif need:
            try:
                ws = torch.empty(need, dtype=torch.uint8, device=dev)
            except torch.OutOfMemoryError:
                need = 0
    _call("bfp_gemm_fp8", dev, *A._ptrs, *B._ptrs, M, N, K, C.data_ptr(), TYPES[C.dtype], ldc,
          ws.data_ptr() if ws is not None else None, need if ws is not None else 0)
    return C


# ---- the norm -----------------------------------------------------------


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: torch.Tensor | None = None, eps: float = 1e-6, to=None,
             rounding: str = "nearest", seed: int = 0, save: bool = False, h_out: torch.Tensor | None = None,
             out=None, status: torch.Tensor | None = None):
    """The root-mean-square norm of x's rows (its last axis, at most 16384 values; the
    leading axes are the rows) with a residual's addition in front: ``(y, h, rstd)`` with
    h = x + residual (without one, x, or x in FP32 where it is BF16 and save is set), rstd
    = (mean(h^2) + eps)^(-1/2) and y = h * rstd * weight, computed in 64 bits and rounded
    once.

    to        None: y in FP32, of x's shape; "e4m3" or "e5m2": an FP8Tensor; 1 .. 8: a
              BFPTensor of that width in groups of 16 (``rounding`` and ``seed`` as
              quantize's).  Converted, y is byte for byte the conversion of the FP32 one.
    save      whether rstd (FP32 [rows]) is written, for rms_norm_grad; else it is None.
    x         FP32 or BF16 (h is FP32 either way; y as well).
    h_out     where h goes; residual or an FP32 x: in place.
    out       a preallocated y.  An FP32 one may be an FP32 x or residual, where h is not: in
              place (without a residual, h is then a copy of x).
    status    as quantize's, of the converted y."""
    xt = _type(x, "x")
    shape = x.shape
    if len(shape) < 1:
        raise ValueError("x must have at least one dimension")
    d = shape[-1]
    rows = shape[0] if len(shape) == 2 else math.prod(shape[:-1])
    dev = x.device
    _f32(weight, "weight", (d,), dev)
    if residual is not None:
        _f32(residual, "residual", shape, dev)
    h = h_out
    if h is not None:
        _f32(h, "h_out", shape, dev)
    elif residual is not None or (xt and save) or (to is None and _same_start(out, x)):
        h = torch.empty_like(x, dtype=torch.float32)
    rstd = None
    if save:  # (the mean of no values: NaN)
        rstd = torch.empty(rows, device=dev, dtype=torch.float32) if d else torch.full((rows,), math.nan, device=dev)
    args = (x.data_ptr(), xt, residual.data_ptr() if residual is not None else None, weight.data_ptr(), rows, d, eps,
            h.data_ptr() if h is not None else None, rstd.data_ptr() if save else None)
    if to is None:
        y = out
        if y is None:
            y = torch.empty_like(x, dtype=torch.float32)
        else:
            _f32(y, "out", shape, dev)
        _call("bfp_rms_norm", dev, *args, y.data_ptr())
    elif isinstance(to, str):
        code, _ = _format(to)
        y = _fp8_out(out, rows, d, to, dev, FP8Tensor.empty)
        _call("bfp_rms_norm_fp8", dev, *args, code, *y._ptrs[:2], _status(status, dev))
    else:
        if rounding not in ROUNDING:
            raise ValueError("rounding must be one of %s" % sorted(ROUNDING))
        y = out if out is not None else BFPTensor.empty(rows, d, 16, to, dev)
        if (y.rows, y.len, y.g, y.m) != (rows, d, 16, to):
            raise ValueError("out has the wrong shape or format")
        _on(dev, out=y.mant)
        _call("bfp_rms_norm_bfp", dev, *args, to, ROUNDING[rounding], seed & 0xFFFFFFFFFFFFFFFF, y.mant.data_ptr(),
              y.exp.data_ptr(), _status(status, dev))
    return y, h if h is not None else x, rstd


@functools.lru_cache(maxsize=4096)
def _norm_grad_ws(rows, d):
    """Workspace bytes of bfp_rms_norm_grad (a function of the sizes alone)."""
    nb = ctypes.c_size_t(0)
    check(load().bfp_rms_norm_grad_ws_size(rows, d, ctypes.byref(nb)), "bfp_rms_norm_grad_ws_size")
    return nb.value


def rms_norm_grad(dy: torch.Tensor, h: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor,
                  dresidual: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """The gradients of rms_norm for dy: ``(dx, dweight)``.  h and rstd are the forward
    pass's (``save=True``); ``dresidual`` is the gradient that reaches h beside the norm,
    added to dx, which is the gradient of x and of the residual alike.  dy is FP32 or BF16,
    the rest FP32.  ``out``: where dx goes; dresidual or an FP32 dy: in place."""
    yt = _type(dy, "dy")
    if dy.dim() < 1:
        raise ValueError("dy must have at least one dimension")
    shape, dev = dy.shape, dy.device
    d = shape[-1]
    rows = shape[0] if len(shape) == 2 else math.prod(shape[:-1])
    _f32(h, "h", shape, dev)
    _f32(rstd, "rstd", (rows,), dev)
    _f32(weight, "weight", (d,), dev)
    if dresidual is not None:
        _f32(dresidual, "dresidual", shape, dev)
    dx = out
    if dx is None:
        dx = torch.empty_like(dy, dtype=torch.float32)
    else:
        _f32(dx, "out", shape, dev)
    need = _norm_grad_ws(rows, d)
    dw, ws = torch.empty(d, dtype=torch.float32, device=dev), torch.empty(need, dtype=torch.uint8, device=dev)
    _call("bfp_rms_norm_grad", dev, dy.data_ptr(), yt, h.data_ptr(), rstd.data_ptr(), weight.data_ptr(),
          dresidual.data_ptr() if dresidual is not None else None, rows, d, dx.data_ptr(), dw.data_ptr(), ws.data_ptr(), need)
    return dx, dw


# ---- the gradients' clipping --------------------------------------------


class TensorList:
    """A list of FP32 (or of BF16) tensors with where their scaled values go (themselves unless ``out``
    is given), checked once: for a program whose gradients stay in place from step to
    step.  It holds their memory (a tensor that is given other memory afterwards, as by
    ``t.data = u``, needs a new list), and a workspace of its own, so calls with one list
    must not overlap, and it lives as long as a graph that was captured with it."""

    def __init__(self, tensors, out=None):
        self.tensors = list(tensors)
        self.out = self.tensors if out is None else list(out)
        if len(self.out) != len(self.tensors):
            raise ValueError("out must have as many tensors as the list")
        n = len(self.tensors)
        self.device = self.tensors[0].device if n and isinstance(self.tensors[0], torch.Tensor) else None
        for name, ts in (("tensors", self.tensors),) + ((("out", self.out),) if out is not None else ()):
            for i, t in enumerate(ts):
                if _type(t, "%s[%d]" % (name, i)) != TYPES[self.tensors[0].dtype]:
                    raise TypeError("%s[%d] must have dtype %s" % (name, i, self.tensors[0].dtype))
                if t.device != self.device:
                    raise ValueError("%s[%d] must be on %s" % (name, i, self.device))
                if t.numel() != self.tensors[i].numel():
                    raise ValueError("out[%d] must have %d values" % (i, self.tensors[i].numel()))
        if n == 0:
            raise ValueError("the list must have a tensor")
        self.type = TYPES[self.tensors[0].dtype]
        self.ptrs = (ctypes.c_void_p * n)(*[t.data_ptr() for t in self.tensors])
        self.out_ptrs = self.ptrs if out is None else (ctypes.c_void_p * n)(*[t.data_ptr() for t in self.out])
        self.sizes = (ctypes.c_int64 * n)(*[t.numel() for t in self.tensors])
        nb = ctypes.c_size_t(0)
        check(load().bfp_sum_squares_ws_size(self.sizes, n, ctypes.byref(nb)), "bfp_sum_squares_ws_size")
        self.pieces = nb.value // 8
        self.work = torch.empty(self.pieces + 1, dtype=torch.float64, device=self.device)  # (and their sum)
        self._memory = [t.detach() for t in (self.tensors if out is None else self.tensors + self.out)]
        self._stream = _stream(self.device)

    def _call(self, name, *args):
        """A call that uses the workspace, which is its own stream's unless that is told."""
        if _stream(self.device) != self._stream:
            self.work.record_stream(torch.cuda.current_stream(self.device))
        _call(name, self.device, *args)

    def __len__(self):
        return len(self.tensors)


def tensor_list(tensors, out=None) -> TensorList:
    """TensorList(tensors, out); ``out``: the tensors that clip_gradients writes to."""
    return TensorList(tensors, out)


def _as_list(tensors):
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def sum_squares(tensors) -> torch.Tensor:
    """The sum of squares over all values of a list of FP32 or BF16 tensors (or a TensorList): one
    float64 value on the card, summed in 64 bits.  Those of several cards or shards are
    added up (all_reduce) before clip_gradients."""
    l = _as_list(tensors)
    out = torch.empty(1, dtype=torch.float64, device=l.device)
    l._call("bfp_sum_squares", l.ptrs, l.type, l.sizes, len(l), out.data_ptr(), l.work.data_ptr(), 8 * l.pieces)
    return out


def clip_gradients(tensors, max_norm: float, sumsq: torch.Tensor | None = None) -> torch.Tensor:
    """Scales a list of FP32 or BF16 tensors (in place; a TensorList: to its ``out``) by min(1,
    max_norm / norm), with norm the root of ``sumsq`` (sum_squares of the list unless one
    is given), and returns norm: one float64 value on the card.  A norm that is infinite
    or NaN scales nothing.  A list that is no TensorList is checked in every call, some
    1 us a tensor on the host."""
    l = _as_list(tensors)
    if not max_norm >= 0.0:
        raise ValueError("max_norm must not be negative")
    if sumsq is None:
        # (a few pieces' sums are added up by the scaling itself)
        pieces = l.pieces
        few = 0 < pieces <= 1024
        at = l.work.data_ptr() if few else l.work.data_ptr() + 8 * pieces
        l._call("bfp_sum_squares", l.ptrs, l.type, l.sizes, len(l), None if few else at, l.work.data_ptr(), 8 * pieces)
        sums = pieces if few else 1
    else:
        _need_cuda(sumsq, "sumsq", torch.float64)
        if sumsq.numel() != 1:
            raise ValueError("sumsq must be one value")
        _on(l.device, sumsq=sumsq)
        at, sums = sumsq.data_ptr(), 1
    norm = torch.empty(1, dtype=torch.float64, device=l.device)
    _call("bfp_clip_gradients", l.device, l.ptrs, l.out_ptrs, l.type, l.sizes, len(l), max_norm, at, sums, norm.data_ptr())
    return norm
