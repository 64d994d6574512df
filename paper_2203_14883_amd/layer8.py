"""Serving a temporal attention layer in 8 bits (Sec. 2.2; node memory and
mailboxes, Sec. 2.1): rows are normed and rounded to 8 bits (``norm_quant``),
projected (``linear_i8``), kept as keys and values of nodes or of their
histories (``cache_write``, ``cache_read``) and attended over
(``cache_attend``).  Argument marshalling only; the kernels are in libtgl
(include/tgl.h has the definitions).

Rounding to 8 bits has no gradient: tensors that require one are refused
while gradients are recorded (use ``torch.no_grad()`` or ``detach()``), and so
are those that carry a forward-mode tangent.  With
``stream``, work is enqueued there and outputs are allocated for it; inputs
made on another stream must be ready, as for every call of the library.
"""
from __future__ import annotations

import ctypes as C
import math
from dataclasses import dataclass, field
from typing import Optional

import torch
from torch.autograd import forward_ad

from .binding import OUT_BF16, OUT_F32, _check, c_cache, c_heads, c_seqs, lib

_TYPES = {torch.float32: OUT_F32, torch.bfloat16: OUT_BF16}
MAX_PAGE = 128
MAX_HEAD_DIM = 256

# A serving step makes many small calls, so the checks below ask a tensor for
# as little as they can (get_device() rather than device, data_ptr() as a plain
# number): 8 to 11 us a call with its outputs, where 11 to 15 were spent before.


def _round16(n: int) -> int:
    return (n + 15) & ~15


def _empty(like: torch.Tensor, shape, dtype, stream) -> torch.Tensor:
    """Memory for a call on that stream (None: the current one)."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _raw_stream(stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _device(t: torch.Tensor, name: str) -> int:
    """The current device, which t has to be on."""
    dev = t.get_device()
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise ValueError("%s must be on the current device, not on %s" % (name, t.device))
    if t.requires_grad or forward_ad._current_level >= 0:
        _no_gradient(t, name)
    return dev


def _also(t: torch.Tensor, name: str, dev: int):
    if t.get_device() != dev:
        raise ValueError("%s must be on the current device, not on %s" % (name, t.device))
    if t.requires_grad or forward_ad._current_level >= 0:
        _no_gradient(t, name)


def _no_gradient(t: torch.Tensor, name: str):
    if (t.requires_grad and torch.is_grad_enabled()) or forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError("%s requires a gradient, and rounding to 8 bits has none" % name)


def _type(dtype, name: str) -> int:
    t = _TYPES.get(dtype)
    if t is None:
        raise ValueError("%s must be float32 or bfloat16" % name)
    return t


def _rows(t: torch.Tensor, name: str):
    """Shape and row stride of a matrix whose rows are contiguous."""
    if t.dim() != 2:
        raise ValueError("%s must be a matrix" % name)
    n, dim = t.shape
    stride, inner = t.stride()
    if inner != 1 and dim > 1 and n > 0:
        raise ValueError("%s must have the elements of a row next to each other" % name)
    return n, dim, stride


def _vector(t: torch.Tensor, n: int, name: str, dev: int, dtype=torch.float32) -> int:
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s vector of %d" % (name, dtype, n))
    _also(t, name, dev)
    return t.data_ptr()


# --------------------------------------------------------------------------
# rows
# --------------------------------------------------------------------------

def _quantise(x, weight, residual, normalize, eps, stream, out):
    dev = _device(x, "x")
    dt = _type(x.dtype, "x")
    n, dim, xs = _rows(x, "x")
    if dim < 1:
        raise ValueError("x must have columns")
    w = None if weight is None else _vector(weight, dim, "weight", dev)
    rs = os = 0
    for t, name in ((residual, "residual"), (out, "out")):
        if t is None:
            continue
        if t.dtype != x.dtype or t.shape != x.shape:
            raise ValueError("%s must have x's type and shape" % name)
        _also(t, name, dev)
        if name == "residual":
            rs = _rows(t, name)[2]
        else:
            os = _rows(t, name)[2]
            if n > 1 and os < dim:
                raise ValueError("out's rows overlap")
    width = _round16(dim)
    store = _empty(x, (n, width), torch.int8, stream)
    scale = _empty(x, (n,), torch.float32, stream)
    if out is None and residual is not None:
        out = _empty(x, (n, dim), x.dtype, stream)
        os = dim
    if n:
        s = lib().tgl_norm_quant(x.data_ptr(), xs, None if residual is None else residual.data_ptr(), rs, w, n, dim, dt,
                                 normalize, eps, store.data_ptr(), width, scale.data_ptr(),
                                 None if out is None else out.data_ptr(), os if os > dim else dim, _raw_stream(stream, dev))
        if s:
            _check(s, "tgl_norm_quant")
    return store if width == dim else store[:, :dim], scale, out


def norm_quant(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
               eps: float = 1e-6, out: Optional[torch.Tensor] = None, stream=None):
    """Residual addition, root-mean-square norm and rounding to 8 bits of rows.

    ``x`` (and ``residual``) are ``[n, dim]`` float32 or bfloat16, ``weight``
    float32 ``[dim]``.  Returns ``(q, scale, h)``: int8 ``[n, dim]`` (rows padded
    with zeros to 16 bytes, as ``linear_i8`` takes them) and float32 ``[n]``, whose
    product is ``h / rms(h) * weight`` for ``h = x + residual``; ``h`` in x's type
    goes to ``out`` (allocated if there is a residual and ``out`` is None; it may
    be ``x`` or ``residual`` itself), or is None."""
    return _quantise(x, weight, residual, True, eps, stream, out)


def quant_rows(x: torch.Tensor, stream=None):
    """Rows rounded to 8 bits: ``(q, scale)`` with ``q * scale`` standing for
    ``x``, a scale per row.  A weight matrix ``[out, in]`` gets its scale per
    output channel this way, once, when it is loaded."""
    q, scale, _ = _quantise(x, None, None, False, 0.0, stream, None)
    return q, scale


def _int8_rows(t: torch.Tensor, name: str, dev: int):
    """Shape and row stride of int8 rows that the kernel can read."""
    if t.dtype != torch.int8:
        raise ValueError("%s must be int8" % name)
    _also(t, name, dev)
    m, k, stride = _rows(t, name)
    if m < 2:
        stride = _round16(k)
    if m and (stride & 15 or t.data_ptr() & 15 or stride < 0
              or (k & 15 and t.storage_offset() + (m - 1) * stride + _round16(k) > t.untyped_storage().nbytes())):
        raise ValueError("%s must have rows at multiples of 16 bytes, padded to 16 bytes (as quant_rows and norm_quant "
                         "make them)" % name)
    return m, k, stride


def linear_i8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
              bias: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16, out: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """``out = (x * x_scale[:, None]) @ (w * w_scale[:, None]).T + bias`` for int8
    ``x [m, k]`` and ``w [n, k]`` with float32 scales per row, bias float32
    ``[n]``; ``[m, n]`` float32 or bfloat16.  The sums are exact.  Rows start at
    multiples of 16 bytes and are readable up to the next one, as
    ``norm_quant`` and ``quant_rows`` leave them."""
    dev = _device(x, "x")
    m, k, xstride = _int8_rows(x, "x", dev)
    n, wk, wstride = _int8_rows(w, "w", dev)
    if wk != k or k < 1 or n < 1:
        raise ValueError("x is %s and w %s: both need the same number of columns" % (tuple(x.shape), tuple(w.shape)))
    xs = _vector(x_scale, m, "x_scale", dev)
    ws = _vector(w_scale, n, "w_scale", dev)
    b = None if bias is None else _vector(bias, n, "bias", dev)
    ostride = n
    if out is not None:
        out_dtype = out.dtype
        _also(out, "out", dev)
        om, on, ostride = _rows(out, "out")
        if om != m or on != n or (m > 1 and ostride < n):
            raise ValueError("out must be [%d, %d]" % (m, n))
    ot = _type(out_dtype, "the output")
    if out is None:
        out = _empty(x, (m, n), out_dtype, stream)
    if m:
        s = lib().tgl_linear_i8(x.data_ptr(), xstride, xs, m, w.data_ptr(), wstride, ws, b, n, k, out.data_ptr(),
                            ostride if ostride > n else n, ot, _raw_stream(stream, dev))
        if s:
            _check(s, "tgl_linear_i8")
    return out


# --------------------------------------------------------------------------
# cache
# --------------------------------------------------------------------------

@dataclass(frozen=True, eq=False)
class HistoryCache:
    """Keys and values in 8 bits, in pages of P tokens: ``data`` int8 ``[pages,
    heads, 2, P, Dp]`` (keys, then values; Dp = dim rounded up to 16) and
    ``scales`` float32 ``[pages, heads, 2]``, one step for a page's keys and one
    for its values per head.  P is a power of two up to 128; P = 1 keeps one
    token per page (a node's memory), so that neighbour ids are page ids."""
    data: torch.Tensor
    scales: torch.Tensor
    dim: int
    _view: c_cache = field(init=False, repr=False, compare=False)

    def __post_init__(self):
        d, s = self.data, self.scales
        if d.dim() != 5 or d.dtype != torch.int8 or not d.is_contiguous():
            raise ValueError("data must be a contiguous int8 tensor [pages, heads, 2, P, Dp]")
        pages, heads, two, P, width = d.shape
        if s.dtype != torch.float32 or not s.is_contiguous() or s.shape != (pages, heads, 2):
            raise ValueError("scales must be a contiguous float32 tensor [pages, heads, 2]")
        if not 1 <= self.dim <= MAX_HEAD_DIM or width != _round16(self.dim) or two != 2 or heads < 1:
            raise ValueError("data must hold keys and values of %d elements padded to 16, at most %d"
                             % (self.dim, MAX_HEAD_DIM))
        if P < 1 or P > MAX_PAGE or P & (P - 1):
            raise ValueError("a page holds 1, 2, 4, ... or %d tokens" % MAX_PAGE)
        if d.get_device() != s.get_device():
            raise ValueError("data and scales must be on the same device")
        object.__setattr__(self, "_view", c_cache(d.data_ptr() if pages else None, s.data_ptr() if pages else None,
                                                  pages, P, heads, self.dim, 0))

    def __reduce__(self):                   # copies and pickles: the view is made anew, of the copy's tensors
        return type(self), (self.data, self.scales, self.dim)

    @classmethod
    def empty(cls, num_pages: int, heads: int, dim: int, page_tokens: int = 1, device="cuda") -> "HistoryCache":
        """A cache of that many pages, zeros everywhere."""
        return cls(torch.zeros((num_pages, heads, 2, page_tokens, _round16(dim)), dtype=torch.int8, device=device),
                   torch.zeros((num_pages, heads, 2), dtype=torch.float32, device=device), dim)

    @property
    def num_pages(self) -> int:
        return int(self._view.num_pages)

    @property
    def heads(self) -> int:
        return int(self._view.heads)

    @property
    def page_tokens(self) -> int:
        return int(self._view.page_tokens)

    def c_view(self) -> c_cache:
        return self._view


def _seqs(dev: int, table, start, offsets, start_name="start") -> c_seqs:
    if table.dtype != torch.int32 or table.dim() != 2:
        raise ValueError("table must be an int32 tensor [sequences, pages]")
    _also(table, "table", dev)
    B, width = table.shape
    stride, inner = table.stride()
    if inner != 1 and width > 1 and B > 0:
        raise ValueError("table must have the pages of a sequence next to each other")
    return c_seqs(table.data_ptr() or None, stride, B, width, 0,
                  None if start is None else _vector(start, B, start_name, dev, torch.int64),
                  None if offsets is None else _vector(offsets, B + 1, "offsets", dev, torch.int64))


def _heads(t: torch.Tensor, name: str, n: int, heads: int, dim: int) -> c_heads:
    if t.dim() != 3 or t.shape != (n, heads, dim):
        raise ValueError("%s must be [%d, %d, %d]" % (name, n, heads, dim))
    token, head, inner = t.stride()
    if inner != 1 and dim > 1 and n > 0:
        raise ValueError("%s must have the elements of a head next to each other" % name)
    return c_heads(t.data_ptr() or None, token, head)


def _apart(t: torch.Tensor, name: str):
    if any(stride == 0 and size > 1 for stride, size in zip(t.stride(), t.shape)):
        raise ValueError("%s's rows overlap" % name)


def _cache_device(cache: HistoryCache) -> int:
    dev = cache.data.get_device()
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise ValueError("the cache must be on the current device")
    _also(cache.scales, "the cache's scales", dev)
    return dev


def _check_shares(n: int, seqs: int):
    if n % seqs if seqs else n:
        raise ValueError("%d tokens do not divide among %d sequences: offsets are needed" % (n, seqs))


def cache_write(cache: HistoryCache, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor,
                start: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None, stream=None) -> None:
    """Appends keys and values ``[tokens, heads, dim]`` to the histories of an
    8-bit cache.  Sequence b (row b of ``table``, int32 page ids, negative =
    padding) gets tokens ``offsets[b]:offsets[b+1]`` at its positions
    ``start[b]`` onwards (int64 device tensors; ``start`` None: 0, ``offsets``
    None: the same number for every sequence, so a new token each for one row
    per sequence).  What a history holds below ``start[b]`` stays; a page that it
    ends in keeps one step for old and new tokens, old ones being rounded
    again when it grows.  A page belongs to one sequence of the call."""
    dev = _cache_device(cache)
    _also(k, "k", dev)
    _also(v, "v", dev)
    if k.dtype != v.dtype:
        raise ValueError("k and v must have the same type")
    dt = _type(k.dtype, "k")
    view = cache._view
    n = k.shape[0]
    sq = _seqs(dev, table, start, offsets)
    if offsets is None:
        _check_shares(n, sq.num_seqs)
    kh, vh = _heads(k, "k", n, view.heads, view.dim), _heads(v, "v", n, view.heads, view.dim)
    s = lib().tgl_cache_write(C.byref(view), C.byref(kh), C.byref(vh), dt, n, C.byref(sq), _raw_stream(stream, dev))
    if s:
        _check(s, "tgl_cache_write")


def cache_read(cache: HistoryCache, table: torch.Tensor, start: Optional[torch.Tensor] = None,
               offsets: Optional[torch.Tensor] = None, n: Optional[int] = None, out_dtype=torch.float32,
               k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None, stream=None):
    """Keys and values of tokens read back from an 8-bit cache, ``[n, heads,
    dim]`` float32 or bfloat16 each; zeros where a place is padding.  Places
    are given as for ``cache_write``; ``n`` (default: every place of the table)
    is the number of tokens, ``offsets[-1]`` where there are offsets.  Tokens that
    no sequence owns are not written."""
    dev = _cache_device(cache)
    view = cache._view
    sq = _seqs(dev, table, start, offsets)
    if n is None:
        n = table.numel() * view.page_tokens
    if offsets is None:
        _check_shares(n, sq.num_seqs)
    if (k is None) != (v is None) or (k is not None and k.dtype != v.dtype):
        raise ValueError("k and v go together, with one type")
    if k is None:
        ot = _type(out_dtype, "the output")
        k = _empty(cache.data, (n, view.heads, view.dim), out_dtype, stream)
        v = _empty(cache.data, (n, view.heads, view.dim), out_dtype, stream)
    else:
        ot = _type(k.dtype, "k")
        _also(k, "k", dev)
        _also(v, "v", dev)
        _apart(k, "k")
        _apart(v, "v")
    kh, vh = _heads(k, "k", n, view.heads, view.dim), _heads(v, "v", n, view.heads, view.dim)
    s = lib().tgl_cache_read(C.byref(view), C.byref(kh), C.byref(vh), ot, n, C.byref(sq), _raw_stream(stream, dev))
    if s:
        _check(s, "tgl_cache_read")
    return k, v


def cache_attend(cache: HistoryCache, q: torch.Tensor, table: torch.Tensor, begin: Optional[torch.Tensor] = None,
                 end: Optional[torch.Tensor] = None, scale: Optional[float] = None, return_lse: bool = False,
                 out: Optional[torch.Tensor] = None, stream=None):
    """Attention of queries over an 8-bit cache.

    ``q`` is ``[B, q_heads, dim]`` (one query per sequence) or ``[B, T, q_heads,
    dim]`` float32 or bfloat16; q_heads is a multiple of the cache's heads, and
    query head h reads head ``h // (q_heads // heads)``.  Query t of sequence b
    sees positions ``begin[b] <= p < end[b] - (T - 1 - t)`` of row b of ``table``
    (int64 device tensors; None: from 0, to the row's end), without padding:
    a table of a node's pages is attention over its history, and the
    neighbour ids of sampled slots over one-token pages is attention over
    the sampled neighbours.  ``scale`` defaults to ``1 / sqrt(dim)``.  Rows that
    see nothing are 0; rows whose largest score is no finite number are NaN.  Queries are held to 2^-24 of their row's largest element and
    weights to 2^-22 of themselves, in either type.  Returns ``out`` like q, and with ``return_lse`` the
    logarithm of each row's sum of exponentials, float32 ``[B(, T), q_heads]``."""
    dev = _cache_device(cache)
    _also(q, "q", dev)
    dt = _type(q.dtype, "q")
    view = cache._view
    heads, dim = view.heads, view.dim
    sq = _seqs(dev, table, begin, None, "begin")
    B = sq.num_seqs
    shape = q.shape
    if len(shape) == 3:
        T = 1
    elif len(shape) == 4:
        T = shape[1]
    else:
        T = 0
    if T < 1 or shape[0] != B or shape[-1] != dim:
        raise ValueError("q must be [%d, heads, %d] or [%d, queries, heads, %d] with at least one query" % (B, dim, B, dim))
    H = shape[-2]
    if H < 1 or H % heads:
        raise ValueError("q has %d heads: a multiple of the cache's %d heads is needed" % (H, heads))
    last = None if end is None else _vector(end, B, "end", dev, torch.int64)
    rows = B * T
    L = lib()
    need = L.tgl_cache_attend_workspace(C.byref(view), C.byref(sq), H, T)
    given = out is not None
    if not given:
        out = _empty(q, shape, q.dtype, stream)
    lse = _empty(q, shape[:-1], torch.float32, stream) if return_lse else None
    ws = _empty(q, (need,), torch.uint8, stream) if need else None
    if given:
        if out.dtype != q.dtype or out.shape != shape:
            raise ValueError("out must have q's type and shape")
        _also(out, "out", dev)
        _apart(out, "out")
    qh, oh = _heads(_flat(q, "q", rows), "q", rows, H, dim), _heads(_flat(out, "out", rows), "out", rows, H, dim)
    s = L.tgl_cache_attend(C.byref(view), C.byref(qh), H, T, dt, C.byref(sq), last,
                           1.0 / math.sqrt(dim) if scale is None else scale, C.byref(oh),
                           None if lse is None else lse.data_ptr() or None, None if ws is None else ws.data_ptr(), need,
                           _raw_stream(stream, dev))
    if s:
        _check(s, "tgl_cache_attend")
    return (out, lse) if return_lse else out


def _flat(t: torch.Tensor, name: str, rows: int) -> torch.Tensor:
    """[B, T, H, D] as [B T, H, D], without a copy."""
    if t.dim() == 3:
        return t
    try:
        return t.view(rows, t.shape[2], t.shape[3])
    except RuntimeError:
        raise ValueError("%s must have its queries at one stride over the sequences" % name) from None
