"""Attention and a cache of keys and values in 4 or 8 bits: ctypes marshalling of the calls, and attention's torch
autograd form.

Queries, keys, values and outputs are [rows, heads, head_dim] in float32, float16 or bfloat16, a row for each token; sequences lie
one after the other, and ``starts`` (int32, on the device, one more than sequences, from 0) says where each begins.  Heads
and rows may be any distance apart (slices of a projection's output), a head's elements are contiguous.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import OUT_INT4, OUT_INT8, _check, _WTYPES, lib
from .linear import _current_stream, _device, _workspace

_SCALE_GROUP = 32  # elements of a head that share a scale in the cache


class squant_heads_t(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row", ctypes.c_int64), ("head", ctypes.c_int64)]


class squant_cache_t(ctypes.Structure):
    _fields_ = [("key_codes", ctypes.c_void_p), ("key_scales", ctypes.c_void_p), ("value_codes", ctypes.c_void_p),
                ("value_scales", ctypes.c_void_p), ("pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("format", ctypes.c_int)]


class squant_paged_t(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("starts", ctypes.c_void_p),
                ("sequences", ctypes.c_int32), ("table_width", ctypes.c_int32)]


class squant_packed_t(ctypes.Structure):
    _fields_ = [("q_starts", ctypes.c_void_p), ("k_starts", ctypes.c_void_p), ("sequences", ctypes.c_int32),
                ("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        L = lib()
        i64, i32, vp, sz, en, fl = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
        hp, cp = ctypes.POINTER(squant_heads_t), ctypes.POINTER(squant_cache_t)
        wp, pp = ctypes.POINTER(squant_paged_t), ctypes.POINTER(squant_packed_t)
        L.squant_cache_write.argtypes = [hp, hp, en, i64, cp, wp, vp]
        L.squant_cache_read.argtypes = [cp, wp, en, i64, hp, hp, vp]
        L.squant_cache_attention_workspace_bytes.argtypes = [i64, i32, cp, wp]
        L.squant_cache_attention.argtypes = [hp, en, i64, i32, cp, wp, fl, hp, vp, sz, vp]
        L.squant_attention_workspace_bytes.argtypes = [pp, en]
        L.squant_attention.argtypes = [hp, hp, hp, en, pp, hp, vp, vp, sz, vp]
        L.squant_attention_backward_workspace_bytes.argtypes = [pp, en]
        L.squant_attention_backward.argtypes = [hp, hp, hp, hp, hp, vp, en, pp, hp, hp, hp, vp, sz, vp]
        for f in ("cache_write", "cache_read", "cache_attention", "attention", "attention_backward"):
            getattr(L, f"squant_{f}").restype = en
        L.squant_cache_attention_workspace_bytes.restype = sz
        L.squant_attention_workspace_bytes.restype = sz
        L.squant_attention_backward_workspace_bytes.restype = sz
        _ready = L
    return _ready


class QuantizedCache(NamedTuple):
    """Keys and values of 4-bit (uint8, two codes a byte) or 8-bit (int8) codes [pages, heads, page_size, head_dim or half of
    it], with a bfloat16 scale [pages, heads, page_size, head_dim / 32] for each 32 of a head's elements."""
    key_codes: torch.Tensor
    key_scales: torch.Tensor
    value_codes: torch.Tensor
    value_scales: torch.Tensor

    @classmethod
    def empty(cls, pages: int, heads: int, page_size: int, head_dim: int, format: int = OUT_INT4, device="cuda") -> "QuantizedCache":
        """A cache whose slots hold nothing yet."""
        if format not in (OUT_INT4, OUT_INT8):
            raise ValueError("format must be OUT_INT4 or OUT_INT8")
        if head_dim not in (32, 64, 96, 128, 192, 256):
            raise ValueError("head_dim must be 32, 64, 96, 128, 192 or 256")
        shape = (pages, heads, page_size)

        def one():
            if format == OUT_INT4:
                codes = torch.empty(shape + (head_dim // 2,), dtype=torch.uint8, device=device)
            else:
                codes = torch.empty(shape + (head_dim,), dtype=torch.int8, device=device)
            return codes, torch.empty(shape + (head_dim // _SCALE_GROUP,), dtype=torch.bfloat16, device=device)
        return cls(*one(), *one())


_HEAD_DIMS = frozenset((32, 64, 96, 128, 192, 256))


def _cache(cache: QuantizedCache, device: int) -> squant_cache_t:
    kc, ks, vc, vs = cache
    shape = kc.shape
    if kc.dtype is torch.uint8:
        fmt, dim = OUT_INT4, 2 * shape[-1] if len(shape) == 4 else 0
    elif kc.dtype is torch.int8:
        fmt, dim = OUT_INT8, shape[-1] if len(shape) == 4 else 0
    else:
        raise ValueError("a cache's codes must be int8, or uint8 with two 4-bit codes a byte")
    if dim not in _HEAD_DIMS:
        raise ValueError("a cache's codes must be [pages, heads, page_size, bytes] of heads of 32, 64, 96, 128, 192 or 256 elements")
    pages, heads, page_size, _ = shape
    scales = (pages, heads, page_size, dim // _SCALE_GROUP)
    if (vc.dtype is not kc.dtype or vc.shape != shape or ks.shape != scales or vs.shape != scales
            or ks.dtype is not torch.bfloat16 or vs.dtype is not torch.bfloat16):
        raise ValueError("a cache's values must be like its keys, its scales bfloat16 with one for each 32 elements")
    if not (kc.is_contiguous() and ks.is_contiguous() and vc.is_contiguous() and vs.is_contiguous()
            and kc.get_device() == ks.get_device() == vc.get_device() == vs.get_device() == device):
        raise ValueError("a cache's tensors must be contiguous and on the activations' device")
    return squant_cache_t(kc.data_ptr(), ks.data_ptr(), vc.data_ptr(), vs.data_ptr(), pages, page_size, heads, dim, fmt)


def _ints(t: torch.Tensor, count: Optional[int], what: str, device: int) -> int:
    if (t.dtype is not torch.int32 or t.dim() != 1 or not t.is_contiguous() or t.get_device() != device
            or (t.shape[0] < 1 if count is None else t.shape[0] != count)):
        raise ValueError(f"{what} must be a contiguous int32 tensor on the activations' device"
                         + (f" of {count} elements" if count is not None else ""))
    return t.data_ptr()


def _paged(table: torch.Tensor, lengths: torch.Tensor, starts: Optional[torch.Tensor], rows: int, device: int) -> squant_paged_t:
    if table.dtype is not torch.int32 or table.dim() != 2 or not table.is_contiguous() or table.get_device() != device:
        raise ValueError("table must be a contiguous int32 tensor [sequences, pages of each] on the activations' device")
    sequences, width = table.shape
    at = _ints(lengths, sequences, "lengths", device)
    if starts is not None:
        return squant_paged_t(table.data_ptr(), at, _ints(starts, sequences + 1, "starts", device), sequences, width)
    if rows != sequences:
        raise ValueError("without starts there must be one row for each sequence")
    return squant_paged_t(table.data_ptr(), at, None, sequences, width)


def _heads(t: torch.Tensor, shape, what: str, device: int, dtype) -> squant_heads_t:
    """t as [rows, heads, head_dim] of this shape."""
    if t.shape != shape:
        raise ValueError(f"{what} must be [{shape[0]}, {shape[1]}, {shape[2]}]")
    if t.dtype is not dtype or t.get_device() != device:
        raise ValueError(f"{what} must have the type and the device of the other activations")
    row, head, element = t.stride()
    rows, heads, dim = shape
    if element != 1 or head < dim or row < dim:
        if (dim > 1 and element != 1) or (heads > 1 and head < dim) or (rows > 1 and row < dim):
            raise ValueError(f"{what} must have contiguous heads that do not overlap")
    return squant_heads_t(t.data_ptr(), row, head)


def _result(t: Optional[torch.Tensor], shape, what: str, device: int, dtype, like: torch.Tensor):
    """(t, or a new tensor like `like`, as [rows, heads, head_dim] that may be written)."""
    rows, heads, dim = shape
    if t is None:
        t = torch.empty(shape, dtype=dtype, device=like.device)
        return t, squant_heads_t(t.data_ptr(), heads * dim, dim)
    h = _heads(t, shape, what, device, dtype)
    if rows > 1 and heads > 1 and h.row < (heads - 1) * h.head + dim and h.head < (rows - 1) * h.row + dim:
        raise ValueError(f"rows and heads of {what} overlap")
    return t, h


def _extent(h: squant_heads_t, shape, size: int):
    rows, heads, dim = shape
    return h.data or 0, (h.data or 0) + ((rows - 1) * h.row + (heads - 1) * h.head + dim) * size if rows and heads else 0


def _disjoint(a: squant_heads_t, a_shape, b: squant_heads_t, b_shape, size: int) -> bool:
    """Whether no byte belongs to both: one ends before the other begins, or both repeat with one step (of rows, or of heads) and
    lie side by side within it, as slices of a buffer do."""
    (a0, a1), (b0, b1) = _extent(a, a_shape, size), _extent(b, b_shape, size)
    if a1 <= b0 or b1 <= a0:
        return True
    for step_a, step_b, inner_a, inner_b, dim in ((a.row, b.row, a.head, b.head, 1), (a.head, b.head, a.row, b.row, 0)):
        if step_a == step_b and step_a > 0:
            shift = (b0 - a0) % (step_a * size)
            if (((a_shape[dim] - 1) * inner_a + a_shape[2]) * size <= shift
                    and shift + ((b_shape[dim] - 1) * inner_b + b_shape[2]) * size <= step_a * size):
                return True
    return False


def _apart(result: squant_heads_t, shape, what: str, size: int, others) -> None:
    """Refuses a result over what is read, or over another result: (name, tensor's heads, shape) each."""
    for name, h, other in others:
        if not _disjoint(result, shape, h, other, size):
            raise ValueError(f"{what} overlaps {name}")


def _same(a: squant_heads_t, b: squant_heads_t) -> bool:
    return (a.data, a.row, a.head) == (b.data, b.row, b.head)


def _apart_from_cache(result: squant_heads_t, shape, what: str, size: int, cache: QuantizedCache) -> None:
    first, last = _extent(result, shape, size)
    for t in cache:
        if first < t.data_ptr() + t.numel() * t.element_size() and t.data_ptr() < last:
            raise ValueError(f"{what} overlaps the cache")


def _shape3(t: torch.Tensor, what: str):
    shape = t.shape
    if len(shape) != 3:
        raise ValueError(f"{what} must be [rows, heads, head_dim]")
    return shape


def squant_cache_write(k: torch.Tensor, v: torch.Tensor, cache: QuantizedCache, table: torch.Tensor, lengths: torch.Tensor,
                       starts: Optional[torch.Tensor] = None, stream=None) -> None:
    """Quantises new tokens' keys and values [rows, heads, head_dim] into their slots of the cache.

    Token t of sequence b is in slot t % page_size of page table[b, t // page_size]; the rows starts[b] to
    starts[b + 1] - 1 are the last of lengths[b] tokens (the lengths count them).  Without starts, one row for each sequence.
    Rows behind the last sequence, and tokens whose page is none, are written nowhere."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_cache_write(k, v, cache, table, lengths, starts)
    device = _device(k, "k")
    c = _cache(cache, device)
    rows = _shape3(k, "k")[0]
    shape, dtype = (rows, c.heads, c.head_dim), k.dtype
    hk = _heads(k, shape, "k", device, dtype)
    hv = _heads(v, shape, "v", device, dtype)
    w = _paged(table, lengths, starts, rows, device)
    _check(_lib().squant_cache_write(hk, hv, _WTYPES[dtype], rows, c, w, _current_stream(device)))


def squant_cache_read(cache: QuantizedCache, table: torch.Tensor, lengths: torch.Tensor, starts: Optional[torch.Tensor], rows: int,
                      dtype: torch.dtype, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                      stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(keys, values) [rows, heads, head_dim] that the cache holds for the last tokens of each sequence, placed as in
    squant_cache_write; rows behind the last sequence are 0, tokens whose page is none NaN."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_cache_read(cache, table, lengths, starts, rows, dtype, k, v)
    device = _device(cache.key_scales, "cache")
    if dtype not in _WTYPES:
        raise ValueError("dtype must be float32, float16 or bfloat16")
    c = _cache(cache, device)
    if rows < 0:
        raise ValueError("rows must not be negative")
    shape = (rows, c.heads, c.head_dim)
    given = (k is not None, v is not None)
    k, hk = _result(k, shape, "k", device, dtype, cache.key_scales)
    v, hv = _result(v, shape, "v", device, dtype, cache.key_scales)
    if all(given):
        _apart(hk, shape, "k", dtype.itemsize, (("v", hv, shape),))
    for there, h, what in zip(given, (hk, hv), "kv"):
        if there:
            _apart_from_cache(h, shape, what, dtype.itemsize, cache)
    w = _paged(table, lengths, starts, rows, device)
    _check(_lib().squant_cache_read(c, w, _WTYPES[dtype], rows, hk, hv, _current_stream(device)))
    return k, v


def squant_cache_attention(q: torch.Tensor, cache: QuantizedCache, table: torch.Tensor, lengths: torch.Tensor,
                           starts: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """Attention of new tokens' queries [rows, heads, head_dim] over the cache, which holds their keys and values already;
    rows are placed as in squant_cache_write, and each sees the tokens up to its own.

    heads is a multiple of the cache's; scale defaults to head_dim ** -0.5.  For one or a few new tokens of each sequence; a whole
    prompt is squant_attention's.  Rows that see nothing are 0, rows behind the last sequence too.  `out` may be q, but
    overlaps it in no other way."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_cache_attention(q, cache, table, lengths, starts, scale, out)
    device = _device(q, "q")
    c = _cache(cache, device)
    dim = c.head_dim
    rows, heads, _ = _shape3(q, "q")
    if heads % c.heads or heads == 0:
        raise ValueError("q must have a multiple of the cache's heads")
    shape, dtype = (rows, heads, dim), q.dtype
    hq = _heads(q, shape, "q", device, dtype)
    w = _paged(table, lengths, starts, rows, device)
    given = out is not None
    out, ho = _result(out, shape, "out", device, dtype, q)
    if given:
        if not _same(ho, hq):
            _apart(ho, shape, "out", dtype.itemsize, (("q", hq, shape),))
        _apart_from_cache(ho, shape, "out", dtype.itemsize, cache)
    L = _lib()
    nbytes = L.squant_cache_attention_workspace_bytes(rows, heads, c, w)
    ws = _workspace(q, nbytes)
    _check(L.squant_cache_attention(hq, _WTYPES[dtype], rows, heads, c, w, dim ** -0.5 if scale is None else scale, ho,
                                    None if ws is None else ws.data_ptr(), nbytes, _current_stream(device)))
    return out


def _packed(q: torch.Tensor, k: torch.Tensor, starts, k_starts, scale, causal, device: int) -> squant_packed_t:
    rows, heads, dim = _shape3(q, "q")
    keys, kv_heads, _ = _shape3(k, "k")
    if dim == 0 or dim % 8 or dim > 256:
        raise ValueError("head_dim must be a multiple of 8 up to 256")
    if kv_heads == 0 or heads == 0 or heads % kv_heads:
        raise ValueError("q must have a multiple of the heads of k")
    if starts is None:
        if k_starts is not None:
            raise ValueError("k_starts without starts")
        qs = ks = None
        sequences = 1
    else:
        qs = _ints(starts, None, "starts", device)
        sequences = starts.shape[0] - 1
        if k_starts is None and keys != rows:
            raise ValueError("without k_starts there must be as many keys as queries")
        ks = qs if k_starts is None else _ints(k_starts, sequences + 1, "k_starts", device)
    scale = dim ** -0.5 if scale is None else float(scale)
    if not (0 <= scale < math.inf):
        raise ValueError("scale must be finite and not negative")
    return squant_packed_t(qs, ks, sequences, rows, keys, heads, kv_heads, dim, bool(causal), scale)


def squant_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None,
                     k_starts: Optional[torch.Tensor] = None, scale: Optional[float] = None, causal: bool = True,
                     out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(out, lse) of attention over whole prompts: q [q_rows, heads, head_dim], k and v [k_rows, kv_heads, head_dim].

    Query head h goes with key head h // (heads / kv_heads).  starts are the sequences' first rows of q (and of k, unless
    k_starts says otherwise), None: one sequence.  causal: a sequence's last row sees all of its keys, the row before it one
    less, and so on.  lse [heads, q_rows] is the float32 log-sum-exp of each row's scores.  Rows that see no key are 0.
    `out` may be q, but overlaps no input otherwise."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_attention(q, k, v, starts, k_starts, scale, causal, out)
    device = _device(q, "q")
    p = _packed(q, k, starts, k_starts, scale, causal, device)
    dtype = q.dtype
    q_shape, k_shape = (p.q_rows, p.heads, p.head_dim), (p.k_rows, p.kv_heads, p.head_dim)
    hq = _heads(q, q_shape, "q", device, dtype)
    hk = _heads(k, k_shape, "k", device, dtype)
    hv = _heads(v, k_shape, "v", device, dtype)
    given = out is not None
    out, ho = _result(out, q_shape, "out", device, dtype, q)
    if given:
        _apart(ho, q_shape, "out", dtype.itemsize, (() if _same(ho, hq) else (("q", hq, q_shape),)) + (("k", hk, k_shape), ("v", hv, k_shape)))
    lse = torch.empty((p.heads, p.q_rows), dtype=torch.float32, device=q.device)
    L, type_ = _lib(), _WTYPES[dtype]
    nbytes = L.squant_attention_workspace_bytes(p, type_)
    ws = _workspace(q, nbytes)
    _check(L.squant_attention(hq, hk, hv, type_, p, ho, lse.data_ptr(), None if ws is None else ws.data_ptr(), nbytes,
                              _current_stream(device)))
    return out, lse


def squant_attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                              lse: torch.Tensor, starts: Optional[torch.Tensor] = None, k_starts: Optional[torch.Tensor] = None,
                              scale: Optional[float] = None, causal: bool = True, dq: Optional[torch.Tensor] = None,
                              dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                              stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dq, dk, dv) of squant_attention for the gradient dout of its output; out and lse are what it returned.  dq, dk and dv
    overlap neither each other nor what is read; slices of one buffer are fine."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return squant_attention_backward(dout, q, k, v, out, lse, starts, k_starts, scale, causal, dq, dk, dv)
    device = _device(q, "q")
    p = _packed(q, k, starts, k_starts, scale, causal, device)
    dtype = q.dtype
    q_shape, k_shape = (p.q_rows, p.heads, p.head_dim), (p.k_rows, p.kv_heads, p.head_dim)
    hq = _heads(q, q_shape, "q", device, dtype)
    hk = _heads(k, k_shape, "k", device, dtype)
    hv = _heads(v, k_shape, "v", device, dtype)
    ho = _heads(out, q_shape, "out", device, dtype)
    hd = _heads(dout, q_shape, "dout", device, dtype)
    if lse.dtype is not torch.float32 or lse.shape != (p.heads, p.q_rows) or not lse.is_contiguous() or lse.get_device() != device:
        raise ValueError("lse must be what squant_attention returned for these rows")
    given = [(what, q_shape if what == "dq" else k_shape) for what, t in (("dq", dq), ("dk", dk), ("dv", dv)) if t is not None]
    dq, gq = _result(dq, q_shape, "dq", device, dtype, q)
    dk, gk = _result(dk, k_shape, "dk", device, dtype, q)
    dv, gv = _result(dv, k_shape, "dv", device, dtype, q)
    if given:
        results = {"dq": gq, "dk": gk, "dv": gv}
        read = [("dout", hd, q_shape), ("q", hq, q_shape), ("k", hk, k_shape), ("v", hv, k_shape), ("out", ho, q_shape)]
        first, last = lse.data_ptr(), lse.data_ptr() + 4 * lse.numel()
        for what, shape in given:
            _apart(results[what], shape, what, dtype.itemsize, read)
            begin, end = _extent(results[what], shape, dtype.itemsize)
            if begin < last and first < end:
                raise ValueError(f"{what} overlaps lse")
            read.append((what, results[what], shape))
    L = _lib()
    nbytes = L.squant_attention_backward_workspace_bytes(p, _WTYPES[dtype])
    ws = _workspace(q, nbytes)
    _check(L.squant_attention_backward(hd, hq, hk, hv, ho, lse.data_ptr(), _WTYPES[dtype], p, gq, gk, gv,
                                       None if ws is None else ws.data_ptr(), nbytes, _current_stream(device)))
    return dq, dk, dv


def _headwise(t: torch.Tensor) -> torch.Tensor:
    """t itself where the calls take it, else a contiguous copy (expanded gradients, transposed views)."""
    stride, shape = t.stride(), t.shape
    if len(shape) == 3 and stride[2] == 1 and stride[1] >= shape[2] and stride[0] >= shape[2]:
        return t
    return t.contiguous()


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, starts, k_starts, scale, causal):
        q, k, v = _headwise(q), _headwise(k), _headwise(v)
        out, lse = squant_attention(q, k, v, starts, k_starts, scale, causal)
        ctx.scale, ctx.causal = scale, causal
        ctx.save_for_backward(q, k, v, out, lse, starts, k_starts)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, starts, k_starts = ctx.saved_tensors
        dq, dk, dv = squant_attention_backward(_headwise(dout), q, k, v, out, lse, starts, k_starts, ctx.scale, ctx.causal)
        need = ctx.needs_input_grad
        return dq if need[0] else None, dk if need[1] else None, dv if need[2] else None, None, None, None, None


def _leaves(*tensors):
    """The nodes that add to the gradients of those which are leaves.  Autograd keeps one for a leaf while any graph uses it, on the
    stream of its first use: a backward pass that is captured while an eager graph holds that node waits on a stream outside
    the capture, which ends the process.  Nodes that an eager call here uses are marked; a captured call refuses them."""
    nodes = [torch.autograd.graph.get_gradient_edge(t).node for t in tensors if t.requires_grad and t.is_leaf]
    if nodes and torch.cuda.is_current_stream_capturing():
        if any("squant_eager" in node.metadata for node in nodes):
            raise RuntimeError("a graph of these leaves that was built outside the capture is still alive: release its outputs first")
    else:
        for node in nodes:
            node.metadata["squant_eager"] = True
    return nodes


def packed_attention(q, k, v, starts=None, k_starts=None, scale: Optional[float] = None, causal: bool = True) -> torch.Tensor:
    """squant_attention's output with gradients for q, k and v.

    For a captured step, forward and backward are captured together, and no graph of the same leaves from outside the capture
    may be alive then: where q, k or v themselves are such leaves of an earlier call, this is refused."""
    nodes = _leaves(q, k, v) if torch.is_grad_enabled() else None  # alive until the graph holds them
    return _Attention.apply(q, k, v, starts, k_starts, scale, causal)
