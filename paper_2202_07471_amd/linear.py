"""Operators on quantised layers: ctypes marshalling of the calls that multiply by the solver's codes, and their
torch autograd forms.

``codes`` and ``scales`` are what ``squant_quantize`` (int8) or ``squant_quantize_ex`` with ``OUT_INT4`` (uint8, two
codes a byte) return: a weight [cout, cin], or a convolution's [cout, cin, kh, kw] taken as [cout, cin * kh * kw].
"""
from __future__ import annotations

import ctypes
from functools import lru_cache
from typing import Optional

import torch

from .binding import OUT_INT4, OUT_INT8, SQuantError, _check, _raw_stream, _stream_ptr, _WTYPES, lib  # noqa: F401

ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "silu": ACT_SILU}
KEEP_NONE, KEEP_INT8, KEEP_FULL = 0, 1, 2
KEEPS = {"none": KEEP_NONE, "int8": KEEP_INT8, "full": KEEP_FULL}
IGNORE_INDEX = -100
_MAX_STRIDE = 1 << 22  # elements between rows that are read as they are
_KEPT_GROUP = 64  # columns of a row that share a scale of the kept pre-activation


class squant_codes_t(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("cout", ctypes.c_int32),
                ("cin", ctypes.c_int32), ("format", ctypes.c_int)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = lib()
        i64, vp, sz, en = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        cp = ctypes.POINTER(squant_codes_t)
        L.squant_linear.argtypes = [vp, i64, en, i64, cp, vp, en, vp, i64, vp, i64, en, vp, vp, vp, sz, vp]
        L.squant_linear_backward.argtypes = [vp, i64, en, i64, cp, en, en, vp, vp, vp, i64, vp, vp, sz, vp]
        L.squant_cross_entropy.argtypes = [vp, i64, en, i64, cp, vp, i64, vp, vp, vp, sz, vp]
        L.squant_cross_entropy_backward.argtypes = [vp, i64, en, i64, cp, vp, i64, vp, vp, vp, i64, vp, sz, vp]
        L.squant_linear_workspace_bytes.argtypes = [vp, i64, en, i64, cp, en]
        L.squant_linear_backward_workspace_bytes.argtypes = [en, i64, cp]
        L.squant_cross_entropy_workspace_bytes.argtypes = [vp, i64, en, i64, cp]
        L.squant_cross_entropy_backward_workspace_bytes.argtypes = [vp, i64, en, i64, cp]
        for f in ("linear", "linear_backward", "cross_entropy", "cross_entropy_backward"):
            getattr(L, f"squant_{f}").restype = en
            getattr(L, f"squant_{f}_workspace_bytes").restype = sz
        _ready = L
    return _ready


@lru_cache(maxsize=4096)
def _workspace_bytes(call: str, aligned, codes_aligned, type_: int, rows: int, cout: int, cin: int, fmt: int,
                     *rest: int) -> int:
    # the size depends on the shapes and on whether rows and codes are aligned to 16 bytes: addresses that stand for both
    w = squant_codes_t(256 if codes_aligned else 257, 256, cout, cin, fmt)
    x = () if aligned is None else (256, -(-cin // 8) * 8) if aligned else (256, cin | 1)
    return int(getattr(_lib(), f"squant_{call}_workspace_bytes")(*x, type_, rows, ctypes.byref(w), *rest))


def _workspace(x: torch.Tensor, nbytes: int) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device=x.device) if nbytes else None


def _aligned(t: torch.Tensor, ld: int) -> bool:
    """Whether the products read 16-bit rows as they are, if their length allows it."""
    return (ld | t.data_ptr() >> 1) & 7 == 0 and ld <= _MAX_STRIDE


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _current_stream(device: int) -> int:
    return int(_raw_stream(device)) if _raw_stream is not None else _stream_ptr(None)


def _device(t: torch.Tensor, what: str) -> int:
    """The index of t's device, which has to be the current one."""
    device = t.get_device()  # -1 on the host
    if device < 0 or t.dtype not in _WTYPES:
        raise ValueError(f"{what} must be a float32, float16 or bfloat16 tensor in device memory")
    if device != _current_device():
        raise ValueError(f"{what} is not on the current device")
    return device


def _rows(t: torch.Tensor, cols: int, what: str):
    """(rows, elements between rows) of an activation tensor whose last dimension is `cols`."""
    shape, stride = t.shape, t.stride()
    n = len(shape)
    if n == 0 or shape[-1] != cols or cols == 0:
        raise ValueError(f"{what} must have {cols or 'some'} elements in its last dimension")
    if cols > 1 and stride[-1] != 1:
        raise ValueError(f"{what} must be contiguous in its last dimension")
    if n == 2:
        rows = shape[0]
        ld = stride[0] if rows > 1 else cols
        if ld < cols:
            raise ValueError(f"rows of {what} overlap")
        return rows, ld
    if n == 1:
        return 1, cols
    if not t.is_contiguous():
        raise ValueError(f"{what} of more than two dimensions must be contiguous")
    return t.numel() // cols, cols


def _like(t: torch.Tensor, cols: int, what: str, like: torch.Tensor, device: int) -> int:
    """Elements between the rows of an activation tensor that goes with `like`."""
    shape, other = t.shape, like.shape
    if t.dtype is not like.dtype or t.get_device() != device or shape[:-1] != other[:-1]:
        raise ValueError(f"{what} must have the type, the device and the leading dimensions of the other activations")
    if shape[-1:] == (cols,) and t.is_contiguous():
        return cols
    return _rows(t, cols, what)[1]


def _codes(codes: torch.Tensor, scales: torch.Tensor, cin: int, device: int) -> squant_codes_t:
    if codes.dtype is torch.int8:
        fmt, row = OUT_INT8, cin
    elif codes.dtype is torch.uint8:
        fmt, row = OUT_INT4, (cin + 1) // 2
    else:
        raise ValueError("codes must be int8, or uint8 with two 4-bit codes a byte")
    cout = codes.shape[0] if codes.dim() else 0
    if cin <= 0 or cout <= 0 or codes.numel() != cout * row or not codes.is_contiguous():
        raise ValueError(f"codes must be contiguous with {row} bytes for each of their output channels")
    if scales.dtype is not torch.float32 or scales.shape != (cout,) or not scales.is_contiguous():
        raise ValueError("scales must be a contiguous float32 tensor with one scale for each output channel")
    if codes.get_device() != device or scales.get_device() != device:
        raise ValueError("codes and scales must be on the activations' device")
    return squant_codes_t(codes.data_ptr(), scales.data_ptr(), cout, cin, fmt)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def squant_linear(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, bias: Optional[torch.Tensor] = None,
                  act: int = ACT_NONE, residual: Optional[torch.Tensor] = None, keep: Optional[int] = None,
                  out: Optional[torch.Tensor] = None, stream=None):
    """act(x @ (codes * scales).T + bias) + residual for x [..., cin]; returns [..., cout] of x's type.

    With `keep` (KEEP_INT8, KEEP_FULL or KEEP_NONE) returns (y, kept): the pre-activation for
    squant_linear_backward as (int8 codes, scales), as a tensor of x's type, or None.  `out` may be `residual` and
    may not overlap anything else that is read.
    Asynchronous on `stream` (default: torch's current stream), which the outputs and the workspace belong to."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_linear(x, codes, scales, bias, act, residual, keep, out)
    cin = x.shape[-1] if x.dim() else 0
    device = _device(x, "x")
    rows, ldx = _rows(x, cin, "x")
    w = _codes(codes, scales, cin, device)
    cout = w.cout
    shape = x.shape[:-1] + (cout,)
    if bias is not None and (bias.dtype != x.dtype or bias.shape != (cout,) or not bias.is_contiguous()
                             or bias.get_device() != device):
        raise ValueError("bias must be contiguous, of x's type and device, with one element for each output channel")
    ldr = ldy = cout
    if residual is not None:
        ldr = _like(residual, cout, "residual", x, device)
    if out is None:
        out = x.new_empty(shape)
    else:
        ldy = _like(out, cout, "out", x, device)
        at = out.data_ptr()
        if rows and (at == x.data_ptr() or (residual is not None and at == residual.data_ptr() and ldy != ldr)):
            raise ValueError("out may not lie over x, nor over residual with another distance between rows")
    kept = kept_scales = None
    how = KEEP_NONE if keep is None else keep
    if how == KEEP_INT8:
        kept = torch.empty(shape, dtype=torch.int8, device=x.device)
        kept_scales = torch.empty(x.shape[:-1] + (-(-cout // _KEPT_GROUP),), dtype=torch.float32, device=x.device)
    elif how == KEEP_FULL:
        kept = torch.empty(shape, dtype=x.dtype, device=x.device)
    type_ = _WTYPES[x.dtype]
    nbytes = _workspace_bytes("linear", _aligned(x, ldx), w.codes & 15 == 0, type_, rows, cout, cin, w.format, how)
    ws = _workspace(x, nbytes)
    _check(_lib().squant_linear(x.data_ptr(), ldx, type_, rows, ctypes.byref(w), _ptr(bias), act, _ptr(residual), ldr,
                                out.data_ptr(), ldy, how, _ptr(kept), _ptr(kept_scales), _ptr(ws), nbytes,
                                _current_stream(device)))
    if keep is None:
        return out
    return out, ((kept, kept_scales) if how == KEEP_INT8 else kept)


def squant_linear_backward(dy: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, cin: int, act: int = ACT_NONE,
                           kept=None, bias: bool = True, dx: Optional[torch.Tensor] = None, stream=None):
    """(dx, dbias) of squant_linear for dy [..., cout], codes and scales held fixed; dbias is None without `bias`.

    `kept` is what squant_linear returned beside y.  The residual's gradient is dy."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_linear_backward(dy, codes, scales, cin, act, kept, bias, dx)
    cout = codes.shape[0] if codes.dim() else 0
    device = _device(dy, "dy")
    rows, lddy = _rows(dy, cout, "dy")
    w = _codes(codes, scales, cin, device)
    how, z, z_scales = KEEP_NONE, None, None
    if isinstance(kept, (tuple, list)):
        how, (z, z_scales) = KEEP_INT8, kept
        groups = dy.shape[:-1] + (-(-cout // _KEPT_GROUP),)
        if (z.dtype != torch.int8 or z.shape != dy.shape or not z.is_contiguous() or z.get_device() != device
                or z_scales.dtype != torch.float32 or z_scales.shape != groups or not z_scales.is_contiguous()
                or z_scales.get_device() != device):
            raise ValueError("kept must be the pair that squant_linear returned for these rows")
    elif kept is not None:
        how, z = KEEP_FULL, kept
        if z.dtype != dy.dtype or z.shape != dy.shape or not z.is_contiguous() or z.get_device() != device:
            raise ValueError("kept must be the tensor that squant_linear returned for these rows")
    shape = dy.shape[:-1] + (cin,)
    lddx = cin
    if dx is None:
        dx = dy.new_empty(shape)
    else:
        lddx = _like(dx, cin, "dx", dy, device)
    dbias = dy.new_empty(cout) if bias else None
    type_ = _WTYPES[dy.dtype]
    nbytes = _workspace_bytes("linear_backward", None, w.codes & 15 == 0, type_, rows, cout, cin, w.format)
    ws = _workspace(dy, nbytes)
    _check(_lib().squant_linear_backward(dy.data_ptr(), lddy, type_, rows, ctypes.byref(w), act, how, _ptr(z),
                                         _ptr(z_scales), dx.data_ptr(), lddx, _ptr(dbias), _ptr(ws), nbytes,
                                         _current_stream(device)))
    return dx, dbias


def _check_per_row(t: torch.Tensor, dtype, h: torch.Tensor, what: str):
    if t.dtype != dtype or t.shape != h.shape[:-1] or not t.is_contiguous() or t.get_device() != h.get_device():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor with one element for each row of h")


def squant_cross_entropy(h: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, labels: torch.Tensor,
                         ignore_index: int = IGNORE_INDEX, stream=None):
    """(loss, lse), float32 for each row of h [..., cin], of the logits h @ (codes * scales).T against int64 labels.

    The logits are never in memory.  loss is 0 where the label is `ignore_index` and NaN where it is no entry of
    the vocabulary."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_cross_entropy(h, codes, scales, labels, ignore_index)
    cin = h.shape[-1] if h.dim() else 0
    device = _device(h, "h")
    rows, ldh = _rows(h, cin, "h")
    w = _codes(codes, scales, cin, device)
    _check_per_row(labels, torch.int64, h, "labels")
    loss = torch.empty(h.shape[:-1], dtype=torch.float32, device=h.device)
    lse = torch.empty_like(loss)
    type_ = _WTYPES[h.dtype]
    nbytes = _workspace_bytes("cross_entropy", _aligned(h, ldh), w.codes & 15 == 0, type_, rows, w.cout, cin, w.format)
    ws = _workspace(h, nbytes)
    _check(_lib().squant_cross_entropy(h.data_ptr(), ldh, type_, rows, ctypes.byref(w), labels.data_ptr(),
                                       ignore_index, loss.data_ptr(), lse.data_ptr(), _ptr(ws), nbytes,
                                       _current_stream(device)))
    return loss, lse


def squant_cross_entropy_backward(h: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, labels: torch.Tensor,
                                  lse: torch.Tensor, dloss: torch.Tensor, ignore_index: int = IGNORE_INDEX,
                                  dh: Optional[torch.Tensor] = None, stream=None):
    """dh of squant_cross_entropy for the losses' gradients dloss (float32, one for each row).

    The workspace holds the probabilities of a piece of the vocabulary in 16 bits (float32: 32): about 256 MB, or 4096
    entries of each row where that is more."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_cross_entropy_backward(h, codes, scales, labels, lse, dloss, ignore_index, dh)
    cin = h.shape[-1] if h.dim() else 0
    device = _device(h, "h")
    rows, ldh = _rows(h, cin, "h")
    w = _codes(codes, scales, cin, device)
    _check_per_row(labels, torch.int64, h, "labels")
    _check_per_row(lse, torch.float32, h, "lse")
    _check_per_row(dloss, torch.float32, h, "dloss")
    lddh = cin
    if dh is None:
        dh = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    else:
        lddh = _like(dh, cin, "dh", h, device)
    type_ = _WTYPES[h.dtype]
    nbytes = _workspace_bytes("cross_entropy_backward", _aligned(h, ldh), w.codes & 15 == 0, type_, rows, w.cout, cin, w.format)
    ws = _workspace(h, nbytes)
    _check(_lib().squant_cross_entropy_backward(h.data_ptr(), ldh, type_, rows, ctypes.byref(w), labels.data_ptr(),
                                                ignore_index, lse.data_ptr(), dloss.data_ptr(), dh.data_ptr(), lddh,
                                                _ptr(ws), nbytes, _current_stream(device)))
    return dh


def _rowwise(t: torch.Tensor) -> torch.Tensor:
    """t itself where the calls take it, else a contiguous copy (expanded gradients, transposed views)."""
    if t.is_contiguous() or (t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]):
        return t
    return t.contiguous()


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, codes, scales, bias, act, residual, keep):
        ctx.act, ctx.cin = act, x.shape[-1]
        needed = ctx.needs_input_grad[0] or ctx.needs_input_grad[3]
        how = keep if act != ACT_NONE and needed else KEEP_NONE
        y, kept = squant_linear(_rowwise(x), codes, scales, bias, act,
                                None if residual is None else _rowwise(residual), keep=how)
        ctx.pair = isinstance(kept, tuple)
        ctx.save_for_backward(codes, scales, *(kept if ctx.pair else (kept,)))
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        dx = dbias = None
        if ctx.needs_input_grad[0] or ctx.needs_input_grad[3]:
            codes, scales, *kept = ctx.saved_tensors
            dx, dbias = squant_linear_backward(_rowwise(dy), codes, scales, ctx.cin, ctx.act,
                                               kept if ctx.pair else kept[0], bias=ctx.needs_input_grad[3])
        return (dx if ctx.needs_input_grad[0] else None, None, None, dbias, None,
                dy if ctx.needs_input_grad[5] else None, None)


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, codes, scales, labels, ignore_index):
        h = _rowwise(h)
        loss, lse = squant_cross_entropy(h, codes, scales, labels, ignore_index)
        ctx.ignore_index = ignore_index
        ctx.save_for_backward(h, codes, scales, labels, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        h, codes, scales, labels, lse = ctx.saved_tensors
        return (squant_cross_entropy_backward(h, codes, scales, labels, lse, dloss.contiguous(), ctx.ignore_index),
                None, None, None, None)


def quantized_linear(x, codes, scales, bias=None, act: int = ACT_NONE, residual=None, keep: int = KEEP_INT8):
    """squant_linear with gradients for x, bias and residual; the pre-activation is kept as `keep` says."""
    if act != ACT_NONE and keep not in (KEEP_INT8, KEEP_FULL):
        raise ValueError("keep must be KEEP_INT8 or KEEP_FULL")
    if not torch.is_grad_enabled():  # the function's own needs_input_grad does not tell
        keep = KEEP_NONE
    return _Linear.apply(x, codes, scales, bias, act, residual, keep)


def quantized_cross_entropy(h, codes, scales, labels, ignore_index: int = IGNORE_INDEX):
    """squant_cross_entropy's loss of each row with its gradient for h."""
    return _CrossEntropy.apply(h, codes, scales, labels, ignore_index)
