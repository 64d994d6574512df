"""Serving a temporal attention layer in 8 bits (Sec. 2.2; node memory and
mailboxes, Sec. 2.1): rows are normed and rounded to 8 bits (``norm_quant``),
projected (``linear_i8``), kept as keys and values of nodes or of their
histories (``cache_write``, ``cache_read``) and attended over
(``cache_attend``).  Argument marshalling only; the kernels are in libtgl
(include/tgl.h has the definitions).

Rounding to 8 bits has no gradient: tensors that require one are refused
while gradients are recorded (use ``torch.no_grad()`` or ``detach()``).  With
``stream``, work is enqueued there and outputs are allocated for it; inputs
made on another stream must be ready, as for every call of the library.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math
from dataclasses import dataclass
from typing import Optional

import torch

from .binding import (OUT_BF16, OUT_F32, _check, _p, _stream, c_cache, c_heads, c_seqs, lib)

_TYPES = {torch.float32: OUT_F32, torch.bfloat16: OUT_BF16}
MAX_PAGE = 128
MAX_HEAD_DIM = 256


def _round16(n: int) -> int:
    return (n + 15) // 16 * 16


def _on(stream):
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _checked(device, **tensors):
    """Every tensor is on the current device and records no gradient."""
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda or t.device != device:
            raise ValueError("%s must be on %s, not on %s" % (name, device, t.device))
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError("%s requires a gradient, and rounding to 8 bits has none" % name)


def _device(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.device.index != torch.cuda.current_device():
        raise ValueError("%s must be on the current device" % name)
    return t.device


def _type(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _TYPES:
        raise ValueError("%s must be float32 or bfloat16" % name)
    return _TYPES[t.dtype]


def _out_type(dtype) -> int:
    if dtype not in _TYPES:
        raise ValueError("out_dtype must be float32 or bfloat16")
    return _TYPES[dtype]


def _rows(t: torch.Tensor, name: str, dim: Optional[int] = None):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1 and t.numel() > 0) or (dim is not None and t.shape[1] != dim):
        raise ValueError("%s must be rows%s, adjacent elements next to each other"
                         % (name, "" if dim is None else " of %d" % dim))


def _vector(t: Optional[torch.Tensor], n: int, name: str, dtype=torch.float32):
    if t is not None and (t.dim() != 1 or t.shape[0] != n or t.dtype != dtype or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s vector of %d" % (name, dtype, n))


# --------------------------------------------------------------------------
# rows
# --------------------------------------------------------------------------

def _quantise(x, weight, residual, normalize, eps, stream, out):
    dev = _device(x, "x")
    _checked(dev, x=x, weight=weight, residual=residual, out=out)
    dt = _type(x, "x")
    _rows(x, "x")
    n, dim = x.shape
    if dim < 1:
        raise ValueError("x must have columns")
    _vector(weight, dim, "weight")
    for t, name in ((residual, "residual"), (out, "out")):
        if t is not None:
            if t.dtype != x.dtype or t.shape != x.shape:
                raise ValueError("%s must have x's type and shape" % name)
            _rows(t, name)
    if out is not None and n > 1 and out.stride(0) < dim:
        raise ValueError("out's rows overlap")
    with _on(stream):
        store = torch.empty((n, _round16(dim)), dtype=torch.int8, device=dev)
        scale = torch.empty(n, dtype=torch.float32, device=dev)
        if out is None and residual is not None:
            out = torch.empty((n, dim), dtype=x.dtype, device=dev)
    s = lib().tgl_norm_quant(_p(x) if n else None, x.stride(0), _p(residual) if n else None,
                             0 if residual is None else residual.stride(0), _p(weight), n, dim, dt, int(normalize),
                             C.c_float(eps), _p(store) if n else None, store.stride(0), _p(scale) if n else None,
                             _p(out) if n else None, 0 if out is None else max(out.stride(0), dim), _stream(stream))
    _check(s, "tgl_norm_quant")
    return store[:, :dim], scale, out


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


def _int8_rows(t: torch.Tensor, name: str):
    """Checks int8 rows for the kernel."""
    if t.dtype != torch.int8:
        raise ValueError("%s must be int8" % name)
    _rows(t, name)
    m, k = t.shape
    if m == 0:
        return
    stride = t.stride(0) if m > 1 else _round16(k)
    end = t.storage_offset() + (m - 1) * stride + _round16(k)
    if stride % 16 == 0 and t.data_ptr() % 16 == 0 and stride >= 0 and end <= t.untyped_storage().nbytes():
        return
    raise ValueError("%s must have rows at multiples of 16 bytes, padded to 16 bytes (as quant_rows and norm_quant "
                     "make them)" % name)


def linear_i8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
              bias: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16, out: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """``out = (x * x_scale[:, None]) @ (w * w_scale[:, None]).T + bias`` for int8
    ``x [m, k]`` and ``w [n, k]`` with float32 scales per row, bias float32
    ``[n]``; ``[m, n]`` float32 or bfloat16.  The sums are exact.  Rows start at
    multiples of 16 bytes and are readable up to the next one, as
    ``norm_quant`` and ``quant_rows`` leave them."""
    dev = _device(x, "x")
    _checked(dev, x=x, x_scale=x_scale, w=w, w_scale=w_scale, bias=bias, out=out)
    _int8_rows(x, "x")
    _int8_rows(w, "w")
    m, k = x.shape
    n = w.shape[0]
    if w.shape[1] != k or k < 1 or n < 1:
        raise ValueError("x is %s and w %s: both need the same number of columns" % (tuple(x.shape), tuple(w.shape)))
    _vector(x_scale, m, "x_scale")
    _vector(w_scale, n, "w_scale")
    _vector(bias, n, "bias")
    if out is not None:
        out_dtype = out.dtype
        _rows(out, "out", n)
        if out.shape[0] != m or (m > 1 and out.stride(0) < n):
            raise ValueError("out must be [%d, %d]" % (m, n))
    ot = _out_type(out_dtype)
    L = lib()
    need = int(L.tgl_linear_i8_workspace(m, n, k))
    with _on(stream):
        if out is None:
            out = torch.empty((m, n), dtype=out_dtype, device=dev)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    s = L.tgl_linear_i8(_p(x) if m else None, x.stride(0) if m > 1 else _round16(k), _p(x_scale) if m else None, m,
                        _p(w), w.stride(0) if n > 1 else _round16(k), _p(w_scale), _p(bias), n, k,
                        _p(out) if m else None, out.stride(0) if m > 1 else n, ot, _p(ws), need, _stream(stream))
    _check(s, "tgl_linear_i8")
    return out


# --------------------------------------------------------------------------
# cache
# --------------------------------------------------------------------------

@dataclass
class HistoryCache:
    """Keys and values in 8 bits, in pages of P tokens: ``data`` int8 ``[pages,
    heads, 2, P, Dp]`` (keys, then values; Dp = dim rounded up to 16) and
    ``scales`` float32 ``[pages, heads, 2]``, one step for a page's keys and one
    for its values per head.  P is a power of two up to 128; P = 1 keeps one
    token per page (a node's memory), so that neighbour ids are page ids."""
    data: torch.Tensor
    scales: torch.Tensor
    dim: int

    def __post_init__(self):
        d, s = self.data, self.scales
        if d.dim() != 5 or d.dtype != torch.int8 or not d.is_contiguous():
            raise ValueError("data must be a contiguous int8 tensor [pages, heads, 2, P, Dp]")
        if s.dtype != torch.float32 or not s.is_contiguous() or tuple(s.shape) != tuple(d.shape[:2]) + (2,):
            raise ValueError("scales must be a contiguous float32 tensor [pages, heads, 2]")
        P = d.shape[3]
        if not 1 <= self.dim <= MAX_HEAD_DIM or d.shape[4] != _round16(self.dim) or d.shape[2] != 2:
            raise ValueError("data must hold keys and values of %d elements padded to 16, at most %d"
                             % (self.dim, MAX_HEAD_DIM))
        if P < 1 or P > MAX_PAGE or P & (P - 1):
            raise ValueError("a page holds 1, 2, 4, ... or %d tokens" % MAX_PAGE)
        if d.device != s.device:
            raise ValueError("data and scales must be on the same device")

    @classmethod
    def empty(cls, num_pages: int, heads: int, dim: int, page_tokens: int = 1, device="cuda") -> "HistoryCache":
        """A cache of that many pages, zeros everywhere."""
        return cls(torch.zeros((num_pages, heads, 2, page_tokens, _round16(dim)), dtype=torch.int8, device=device),
                   torch.zeros((num_pages, heads, 2), dtype=torch.float32, device=device), dim)

    @property
    def num_pages(self) -> int:
        return int(self.data.shape[0])

    @property
    def heads(self) -> int:
        return int(self.data.shape[1])

    @property
    def page_tokens(self) -> int:
        return int(self.data.shape[3])

    def c_view(self) -> c_cache:
        n = self.num_pages
        return c_cache(self.data.data_ptr() if n else None, self.scales.data_ptr() if n else None, n,
                       self.page_tokens, self.heads, self.dim, 0)


def _seqs(dev, table, start, offsets, start_name="start") -> c_seqs:
    _checked(dev, table=table, **{start_name: start, "offsets": offsets})
    if table.dim() != 2 or table.dtype != torch.int32 or (
            table.shape[1] > 1 and table.stride(1) != 1 and table.numel() > 0):
        raise ValueError("table must be an int32 tensor [sequences, pages], adjacent pages next to each other")
    B = int(table.shape[0])
    _vector(start, B, start_name, torch.int64)
    _vector(offsets, B + 1, "offsets", torch.int64)
    return c_seqs(table.data_ptr() if table.numel() else None, table.stride(0), B, int(table.shape[1]), 0,
                  None if start is None else start.data_ptr(), None if offsets is None else offsets.data_ptr())


def _heads(t: torch.Tensor, name: str, n: int, heads: int, dim: int) -> c_heads:
    if t.dim() != 3 or tuple(t.shape) != (n, heads, dim) or (dim > 1 and t.stride(2) != 1 and n > 0):
        raise ValueError("%s must be [%d, %d, %d], adjacent elements next to each other" % (name, n, heads, dim))
    return c_heads(t.data_ptr() if t.numel() else None, t.stride(0), t.stride(1))


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
    dev = _device(cache.data, "the cache")
    _checked(dev, k=k, v=v)
    if k.dtype != v.dtype:
        raise ValueError("k and v must have the same type")
    dt = _type(k, "k")
    n = int(k.shape[0])
    sq = _seqs(dev, table, start, offsets)
    if offsets is None and (n % sq.num_seqs if sq.num_seqs else n):
        raise ValueError("%d tokens do not divide among %d sequences: offsets are needed" % (n, sq.num_seqs))
    kh, vh = _heads(k, "k", n, cache.heads, cache.dim), _heads(v, "v", n, cache.heads, cache.dim)
    view = cache.c_view()
    s = lib().tgl_cache_write(C.byref(view), C.byref(kh), C.byref(vh), dt, n, C.byref(sq), _stream(stream))
    _check(s, "tgl_cache_write")


def cache_read(cache: HistoryCache, table: torch.Tensor, start: Optional[torch.Tensor] = None,
               offsets: Optional[torch.Tensor] = None, n: Optional[int] = None, out_dtype=torch.float32,
               k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None, stream=None):
    """Keys and values of tokens read back from an 8-bit cache, ``[n, heads,
    dim]`` float32 or bfloat16 each; zeros where a place is padding.  Places
    are given as for ``cache_write``; ``n`` (default: every place of the table)
    is the number of tokens, ``offsets[-1]`` where there are offsets.  Tokens that
    no sequence owns are not written."""
    dev = _device(cache.data, "the cache")
    sq = _seqs(dev, table, start, offsets)
    if n is None:
        n = int(table.numel()) * cache.page_tokens
    if offsets is None and (n % sq.num_seqs if sq.num_seqs else n):
        raise ValueError("%d tokens do not divide among %d sequences: offsets are needed" % (n, sq.num_seqs))
    if (k is None) != (v is None) or (k is not None and k.dtype != v.dtype):
        raise ValueError("k and v go together, with one type")
    if k is not None:
        out_dtype = k.dtype
    ot = _out_type(out_dtype)
    if k is None:
        with _on(stream):
            k = torch.empty((n, cache.heads, cache.dim), dtype=out_dtype, device=dev)
            v = torch.empty((n, cache.heads, cache.dim), dtype=out_dtype, device=dev)
    _checked(dev, k=k, v=v)
    kh, vh = _heads(k, "k", n, cache.heads, cache.dim), _heads(v, "v", n, cache.heads, cache.dim)
    view = cache.c_view()
    s = lib().tgl_cache_read(C.byref(view), C.byref(kh), C.byref(vh), ot, n, C.byref(sq), _stream(stream))
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
    see nothing are 0.  Returns ``out`` like q, and with ``return_lse`` the
    logarithm of each row's sum of exponentials, float32 ``[B(, T), q_heads]``."""
    dev = _device(cache.data, "the cache")
    _checked(dev, q=q, end=end, out=out)
    dt = _type(q, "q")
    sq = _seqs(dev, table, begin, None, "begin")
    if q.dim() not in (3, 4) or q.shape[0] != sq.num_seqs or q.shape[-1] != cache.dim:
        raise ValueError("q must be [%d, heads, %d] or [%d, queries, heads, %d]"
                         % (sq.num_seqs, cache.dim, sq.num_seqs, cache.dim))
    T = int(q.shape[1]) if q.dim() == 4 else 1
    H = int(q.shape[-2])
    if H < 1 or H % cache.heads or T < 1:
        raise ValueError("q has %d heads and %d queries: at least one query, and a multiple of the cache's %d heads, "
                         "are needed" % (H, T, cache.heads))
    _vector(end, sq.num_seqs, "end", torch.int64)
    rows = sq.num_seqs * T
    with _on(stream):
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=dev)
        lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=dev) if return_lse else None
    if out.dtype != q.dtype or out.shape != q.shape:
        raise ValueError("out must have q's type and shape")

    def flat(t, name):
        try:
            return t if t.dim() == 3 else t.view(rows, H, cache.dim)
        except RuntimeError:
            raise ValueError("%s must have its queries at one stride over the sequences" % name) from None

    qh = _heads(flat(q, "q"), "q", rows, H, cache.dim)
    oh = _heads(flat(out, "out"), "out", rows, H, cache.dim)
    view = cache.c_view()
    L = lib()
    need = int(L.tgl_cache_attend_workspace(C.byref(view), C.byref(sq), H, T))
    with _on(stream):
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    s = L.tgl_cache_attend(C.byref(view), C.byref(qh), H, T, dt, C.byref(sq), _p(end),
                           C.c_float(1.0 / math.sqrt(cache.dim) if scale is None else scale), C.byref(oh), _p(lse),
                           _p(ws), need, _stream(stream))
    _check(s, "tgl_cache_attend")
    return (out, lse) if return_lse else out
