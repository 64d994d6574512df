"""Training a temporal attention layer (Sec. 2.2) in float32 and bfloat16:
rows of several types (kinds of nodes, kinds of events, snapshots) are grouped
(``group_rows``), multiplied with their type's weights (``linear_typed``), and
normed (``layer_norm``), with gradients.  Argument marshalling only; the kernels are
in libtgl (include/tgl.h has the definitions).

``linear_typed`` and ``layer_norm`` record gradients as torch's own operators do;
``linear_typed_backward`` and ``layer_norm_backward`` compute them in calls of
their own, which is also the form to capture into a graph: while a stream is
captured, recording gradients and going backward through these operators are
refused, since a captured backward pass that meets leaves with a living eager
graph ends the process.  Forward-mode tangents are refused.

With ``stream``, work is enqueued there and outputs are allocated for it (the
backward pass runs there too); inputs made on another stream must be ready, as
for every call of the library.
"""
from __future__ import annotations

import ctypes as C
import math
from dataclasses import dataclass, field
from typing import Optional

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from .binding import _changed, _check, c_row_groups, c_typed_weights, lib
from .layer8 import _apart, _empty, _raw_stream, _rows, _type

MAX_TYPES = 1024
MAX_TYPED_DIM = 65536
MAX_NORM_DIM = 16384


def _device(t: torch.Tensor, name: str) -> int:
    """The current device, which t has to be on."""
    dev = t.get_device()
    if dev < 0 or dev != torch._C._cuda_getDevice():
        raise ValueError("%s must be on the current device, not on %s" % (name, t.device))
    if forward_ad._current_level >= 0:
        _no_tangent(t, name)
    return dev


def _also(t: torch.Tensor, name: str, dev: int):
    if t.get_device() != dev:
        raise ValueError("%s must be on the current device, not on %s" % (name, t.device))
    if forward_ad._current_level >= 0:
        _no_tangent(t, name)


def _no_tangent(t: torch.Tensor, name: str):
    if forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError("%s has a forward-mode tangent, which these operators do not carry" % name)


def _floats(t: Optional[torch.Tensor], shape, name: str, dev: int):
    """Address of a contiguous float32 tensor, or None."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous float32 tensor %s" % (name, list(shape)))
    _also(t, name, dev)
    return t.data_ptr()


def _like(t: torch.Tensor, name: str, n: int, dim: int, dtype, dev: int) -> int:
    """Row stride of a matrix that has to be [n, dim] of that type."""
    if t.dtype != dtype or t.dim() != 2 or t.shape[0] != n or t.shape[1] != dim:
        raise ValueError("%s must be a %s matrix [%d, %d]" % (name, dtype, n, dim))
    _also(t, name, dev)
    return _rows(t, name)[2]


def _output(t: torch.Tensor, name: str, n: int, dim: int, dtype, dev: int) -> int:
    stride = _like(t, name, n, dim, dtype, dev)
    _apart(t, name)
    if n > 1 and stride < dim:
        raise ValueError("%s's rows overlap" % name)
    return stride


def _extent(t: torch.Tensor):
    """Bytes of t that lie next to each other, the distances between such pieces, and bytes from the first to behind the last."""
    e = t.element_size()
    if t.is_contiguous():
        return t.numel() * e, [], t.numel() * e
    steps = [stride * e for stride, size in zip(t.stride()[:-1], t.shape) if size > 1]
    whole = sum((size - 1) * stride for size, stride in zip(t.shape[:-1], t.stride())) + t.shape[-1]
    return t.shape[-1] * e, steps, whole * e


def _separate(out: torch.Tensor, *inputs):
    """Refuses an output whose memory workgroups may still read as one of the inputs (tensor, name).  Pieces that recur at
    multiples of one distance may lie between each other: columns beside columns, every other row."""
    own, steps, whole = _extent(out)
    a = out.data_ptr()
    for t, name in inputs:
        if t is None:
            continue
        b = t.data_ptr()
        if b >= a + whole or (t.is_contiguous() and b + t.nbytes <= a):
            continue
        other, more, all_of = _extent(t)
        if b + all_of <= a:
            continue
        pitch = math.gcd(*steps, *more)
        if not pitch or not own <= (b - a) % pitch <= pitch - other:
            raise ValueError("out shares memory with %s" % name)


def _recorded(*tensors) -> bool:
    """Whether gradients are to be recorded for one of the tensors."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _not_captured():
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("gradients are not recorded or followed while a stream is captured: capture "
                           "linear_typed_backward and layer_norm_backward")


def _on(stream, function, *args):
    """function.apply on that stream (None: the current one), if it is not captured."""
    if stream is None:
        _not_captured()
        return function.apply(*args)
    with torch.cuda.stream(stream):
        _not_captured()
        return function.apply(*args)


# --------------------------------------------------------------------------
# rows by type
# --------------------------------------------------------------------------

@dataclass(frozen=True, eq=False)
class RowGroups:
    """Rows by type: type g has the rows ``order[offsets[g]:offsets[g + 1]]``
    (int64 ``offsets [types + 1]``, int32 ``order [n]``; None: the rows lie in
    their types' order), and what lies from ``offsets[-1]`` on has no type.
    Every row is in ``order`` once, and ``offsets`` starts with 0 and does not decrease;
    neither is checked (kernels stay within the rows whatever they hold)."""
    offsets: torch.Tensor
    order: Optional[torch.Tensor] = None
    _view: Optional[c_row_groups] = field(init=False, repr=False, compare=False, default=None)

    def __post_init__(self):
        f, o = self.offsets, self.order
        if f.dtype != torch.int64 or f.dim() != 1 or not 2 <= f.shape[0] <= MAX_TYPES + 1 or not f.is_contiguous():
            raise ValueError("offsets must be a contiguous int64 vector of 1 to %d types and one more" % MAX_TYPES)
        if o is not None:
            if o.dtype != torch.int32 or o.dim() != 1 or not o.is_contiguous():
                raise ValueError("order must be a contiguous int32 vector")
            if o.get_device() != f.get_device():
                raise ValueError("order and offsets must be on the same device")
            object.__setattr__(self, "_view", c_row_groups(o.data_ptr() or None, f.data_ptr(), o.shape[0], self.num_types, 0))

    def __reduce__(self):                   # copies and pickles: the view is made anew, of the copy's tensors
        return type(self), (self.offsets, self.order)

    @property
    def num_types(self) -> int:
        return self.offsets.shape[0] - 1

    def c_view(self, n: int, dev: int) -> c_row_groups:
        """The groups of a call with n rows."""
        _also(self.offsets, "the groups", dev)
        v = self._view
        if v is None:
            return c_row_groups(None, self.offsets.data_ptr(), n, self.num_types, 0)
        if v.n != n:
            raise ValueError("the groups are of %d rows, not of %d" % (v.n, n))
        return v


def group_rows(types: torch.Tensor, num_types: int, ids: Optional[torch.Tensor] = None, stream=None) -> RowGroups:
    """Rows sorted by their type, stable, as ``linear_typed`` takes them.

    ``types`` int32 or int64 ``[n]`` is the type of each row; with ``ids`` (int32
    ``[n]``, the neighbour ids of sampled slots, say) row i has the type
    ``types[ids[i]]``.  Padding (ids that are negative or beyond ``types``) and types
    outside ``[0, num_types)`` are no type: those rows come last."""
    dev = _device(types, "types")
    if types.dtype not in (torch.int32, torch.int64) or types.dim() != 1 or not types.is_contiguous():
        raise ValueError("types must be a contiguous int32 or int64 vector")
    if not 1 <= num_types <= MAX_TYPES:
        raise ValueError("1 to %d types, not %d" % (MAX_TYPES, num_types))
    n = types.shape[0]
    if ids is not None:
        if ids.dtype != torch.int32 or ids.dim() != 1 or not ids.is_contiguous():
            raise ValueError("ids must be a contiguous int32 vector")
        _also(ids, "ids", dev)
        n = ids.shape[0]
    if n >= 1 << 31:
        raise ValueError("fewer than 2^31 rows, not %d" % n)
    L = lib()
    need = L.tgl_group_rows_workspace(n, num_types)
    order = _empty(types, (n,), torch.int32, stream)
    offsets = _empty(types, (num_types + 1,), torch.int64, stream)
    ws = _empty(types, (need,), torch.uint8, stream) if need else None
    # ids of no rows have no address, and would be taken for none
    s = L.tgl_group_rows(types.data_ptr() or None, int(types.dtype == torch.int64), types.shape[0],
                         None if ids is None else ids.data_ptr() or None, n, num_types, order.data_ptr() or None,
                         offsets.data_ptr(), None if ws is None else ws.data_ptr(), need, _raw_stream(stream, dev))
    if s:
        _check(s, "tgl_group_rows")
    return RowGroups(offsets, order)


# --------------------------------------------------------------------------
# products
# --------------------------------------------------------------------------

def _weights(w: torch.Tensor, groups: RowGroups, dtype, dev: int) -> c_typed_weights:
    if w.dim() != 3 or w.dtype != dtype or w.shape[0] != groups.num_types:
        raise ValueError("w must be a %s tensor [%d types, out, in]" % (dtype, groups.num_types))
    _also(w, "w", dev)
    _, out, k = w.shape
    if not 1 <= out <= MAX_TYPED_DIM or not 1 <= k <= MAX_TYPED_DIM:
        raise ValueError("w must have 1 to %d rows and columns" % MAX_TYPED_DIM)
    of_type, row, inner = w.stride()
    if (inner != 1 and k > 1) or (row < k and out > 1):
        raise ValueError("w must have the elements of a row next to each other, and rows apart")
    return c_typed_weights(w.data_ptr(), of_type, max(row, k), out, k)


def _matrix(x: torch.Tensor, name: str, dim: int, dev: int):
    """Number of rows, row stride and type of a matrix of dim columns."""
    dt = _type(x.dtype, name)
    n, columns, stride = _rows(x, name)
    if columns != dim:
        raise ValueError("%s must have %d columns, not %d" % (name, dim, columns))
    _also(x, name, dev)
    return n, stride, dt


def _linear(x, w, groups, bias, out, stream):
    dev = _device(x, "x")
    wv = _weights(w, groups, x.dtype, dev)
    n, xs, dt = _matrix(x, "x", wv.in_, dev)
    view = groups.c_view(n, dev)
    b = _floats(bias, (groups.num_types, wv.out), "bias", dev)
    given = out is not None
    if not given:
        out = _empty(x, (n, wv.out), x.dtype, stream)
        ys = wv.out
    else:
        ys = _output(out, "out", n, wv.out, x.dtype, dev)
        _separate(out, (x, "x"), (w, "w"), (bias, "bias"), (groups.offsets, "the groups"), (groups.order, "the groups"))
    s = lib().tgl_linear_typed(C.byref(view), x.data_ptr() or None, xs, C.byref(wv), b, out.data_ptr() or None,
                               max(ys, wv.out), dt, _raw_stream(stream, dev))
    if s:
        _check(s, "tgl_linear_typed")
    if given:
        _changed(out)
    return out


def _linear_backward(dy, x, w, groups, need_x, need_w, need_b, stream):
    dev = _device(dy, "dy")
    wv = _weights(w, groups, dy.dtype, dev)
    n, dys, dt = _matrix(dy, "dy", wv.out, dev)
    view = groups.c_view(n, dev)
    L = lib()
    raw = _raw_stream(stream, dev)
    dx = dw = db = None
    if need_w or need_b:
        xs = _like(x, "x", n, wv.in_, dy.dtype, dev)
    if need_x:
        dx = _empty(dy, (n, wv.in_), dy.dtype, stream)
        s = L.tgl_linear_typed_grad_x(C.byref(view), dy.data_ptr() or None, dys, C.byref(wv), dx.data_ptr() or None, wv.in_, dt,
                                      raw)
        if s:
            _check(s, "tgl_linear_typed_grad_x")
    if need_w or need_b:
        need = L.tgl_linear_typed_grad_w_workspace(C.byref(view), wv.out, wv.in_, dt)
        dw = _empty(dy, (groups.num_types, wv.out, wv.in_), dy.dtype, stream)
        if need_b:
            db = _empty(dy, (groups.num_types, wv.out), torch.float32, stream)
        ws = _empty(dy, (need,), torch.uint8, stream) if need else None
        s = L.tgl_linear_typed_grad_w(C.byref(view), dy.data_ptr() or None, dys, x.data_ptr() or None, xs, wv.out, wv.in_,
                                      dw.data_ptr(), None if db is None else db.data_ptr(), dt,
                                      None if ws is None else ws.data_ptr(), need, raw)
        if s:
            _check(s, "tgl_linear_typed_grad_w")
    return dx, dw if need_w else None, db


class _LinearTyped(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, groups):
        ctx.groups = groups
        ctx.save_for_backward(x, w, groups.offsets, groups.order)
        return _linear(x, w, groups, bias, None, None)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        _not_captured()
        x, w, offsets, order = ctx.saved_tensors        # as they were: changed in place since, they raise
        if dy.stride(1) != 1 and dy.shape[1] > 1:
            dy = dy.contiguous()
        need = ctx.needs_input_grad
        return _linear_backward(dy, x, w, ctx.groups, need[0], need[1], need[2], None) + (None,)


def linear_typed(x: torch.Tensor, w: torch.Tensor, groups: RowGroups, bias: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Rows times their type's weights: ``out[i] = w[t] @ x[i] + bias[t]`` for a
    row i of type t, zeros for rows of no type.

    ``x [n, in]`` and ``w [types, out, in]`` are float32 or bfloat16, both of one
    type, which the result ``[n, out]`` has too; ``bias`` is float32 ``[types, out]``.
    Sums are float32.  Gradients go to x, w and bias (not with ``out``, which may share no
    memory with an input)."""
    if _recorded(x, w, bias, out):
        if out is not None:
            raise ValueError("out has no gradient: it must be None where gradients are recorded")
        _device(x, "x")
        return _on(stream, _LinearTyped, x, w, bias, groups)
    return _linear(x, w, groups, bias, out, stream)


def linear_typed_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, groups: RowGroups, bias: bool = False, stream=None):
    """Gradients of ``linear_typed`` for the result's gradient ``dy [n, out]``:
    ``(dx, dw, dbias)`` in x's type, w's type and float32 (None without ``bias``).
    Rows of no type get zeros, types without rows too.  dw is summed in float32 over
    stretches of a type's rows and over those in 64 bits, dbias in 64 bits."""
    with torch.no_grad():
        return _linear_backward(dy, x, w, groups, True, True, bias, stream)


# --------------------------------------------------------------------------
# layer norm
# --------------------------------------------------------------------------

def _norm(x, weight, bias, residual, eps, want_stats, stream):
    dev = _device(x, "x")
    dt = _type(x.dtype, "x")
    n, dim, xs = _rows(x, "x")
    if not 1 <= dim <= MAX_NORM_DIM:
        raise ValueError("x must have 1 to %d columns, not %d" % (MAX_NORM_DIM, dim))
    if not eps >= 0.0:
        raise ValueError("eps must not be negative")
    w, b = _floats(weight, (dim,), "weight", dev), _floats(bias, (dim,), "bias", dev)
    rs = 0 if residual is None else _like(residual, "residual", n, dim, x.dtype, dev)
    y = _empty(x, (n, dim), x.dtype, stream)
    h = x if residual is None else _empty(x, (n, dim), x.dtype, stream)
    stats = _empty(x, (n, 2), torch.float64, stream) if want_stats else None
    if n:
        s = lib().tgl_layer_norm(x.data_ptr(), xs, None if residual is None else residual.data_ptr(), rs, w, b, n, dim, dt, eps,
                                 y.data_ptr(), dim, None if residual is None else h.data_ptr(), dim,
                                 None if stats is None else stats.data_ptr(), _raw_stream(stream, dev))
        if s:
            _check(s, "tgl_layer_norm")
    return y, h, stats


def _norm_backward(dy, h, stats, weight, dh, need_x, need_w, need_b, stream):
    dev = _device(dy, "dy")
    dt = _type(dy.dtype, "dy")
    n, dim, dys = _rows(dy, "dy")
    if not 1 <= dim <= MAX_NORM_DIM:
        raise ValueError("dy must have 1 to %d columns, not %d" % (MAX_NORM_DIM, dim))
    hs = _like(h, "h", n, dim, dy.dtype, dev)
    if stats.dtype != torch.float64 or stats.shape != (n, 2) or not stats.is_contiguous():
        raise ValueError("stats must be a contiguous float64 tensor [%d, 2]" % n)
    _also(stats, "stats", dev)
    w = _floats(weight, (dim,), "weight", dev)
    dhs = 0 if dh is None else _like(dh, "dh", n, dim, dy.dtype, dev)
    dx = _empty(dy, (n, dim), dy.dtype, stream) if need_x else None
    dw = _empty(dy, (dim,), torch.float32, stream) if need_w else None
    db = _empty(dy, (dim,), torch.float32, stream) if need_b else None
    L = lib()
    need = L.tgl_layer_norm_grad_workspace(n, dim) if need_w or need_b else 0
    ws = _empty(dy, (need,), torch.uint8, stream) if need else None
    p = [None if t is None else t.data_ptr() or None for t in (dh, dx, dw, db, ws)]
    s = L.tgl_layer_norm_grad(dy.data_ptr() or None, dys, h.data_ptr() or None, hs, stats.data_ptr() or None, w, p[0], dhs,
                              n, dim, dt, p[1], dim, p[2], p[3], p[4], need, _raw_stream(stream, dev))
    if s:
        _check(s, "tgl_layer_norm_grad")
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps):
        ctx.set_materialize_grads(False)
        y, h, stats = _norm(x, weight, bias, residual, eps, True, None)
        ctx.save_for_backward(h, stats, weight)
        ctx.mark_non_differentiable(stats)
        return (y, stats) if residual is None else (y, stats, h)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, _, dh=None):
        _not_captured()
        h, stats, weight = ctx.saved_tensors
        need = ctx.needs_input_grad
        if dy is None:                      # only the sum was used
            return (dh if need[0] else None, dh if need[1] else None) + (
                torch.zeros_like(weight) if need[2] else None, dh.new_zeros(h.shape[1], dtype=torch.float32) if need[3] else None,
                None)
        if dy.stride(1) != 1 and dy.shape[1] > 1:
            dy = dy.contiguous()
        if dh is not None and dh.stride(1) != 1 and dh.shape[1] > 1:
            dh = dh.contiguous()
        dx, dw, db = _norm_backward(dy, h, stats, weight, dh, need[0] or need[1], need[2], need[3], None)
        return dx if need[0] else None, dx if need[1] else None, dw, db, None


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               residual: Optional[torch.Tensor] = None, eps: float = 1e-5, return_stats: bool = False, stream=None):
    """Residual addition and layer norm of rows: ``y = (h - mean(h)) * rstd *
    weight + bias`` with ``h = x + residual`` and ``rstd = 1 / sqrt(var(h) + eps)``.

    ``x`` (and ``residual``) are ``[n, dim]`` float32 or bfloat16, ``weight`` and
    ``bias`` float32 ``[dim]``.  Returns y in x's type; with a residual ``(y, h)``, h in
    x's type as well (the norm is of h as it is returned); with ``return_stats`` the
    rows' mean and rstd too, float64 ``[n, 2]``, for ``layer_norm_backward``.
    Gradients go to x, residual, weight and bias."""
    if _recorded(x, residual, weight, bias):
        _device(x, "x")
        got = _on(stream, _LayerNorm, x, residual, weight, bias, eps)
        y, stats, h = got if residual is not None else (*got, x)
    else:
        y, h, stats = _norm(x, weight, bias, residual, eps, return_stats, stream)
    out = (y,) if residual is None else (y, h)
    if return_stats:
        out += (stats,)
    return out if len(out) > 1 else y


def layer_norm_backward(dy: torch.Tensor, h: torch.Tensor, stats: torch.Tensor, weight: Optional[torch.Tensor] = None,
                        dh: Optional[torch.Tensor] = None, stream=None):
    """Gradients of ``layer_norm`` for the result's gradient ``dy [n, dim]``:
    ``(dx, dweight, dbias)`` in dy's type and float32.  ``h`` and ``stats`` are what
    ``layer_norm`` returned (h is x without a residual), ``dh`` a gradient that reaches h
    besides, which is added to dx.  dx is the gradient of x and of the residual."""
    with torch.no_grad():
        return _norm_backward(dy, h, stats, weight, dh, True, True, True, stream)
