"""The C ABI and the binding of the training operators: what they refuse before
they touch the device (every call here fails a host check, or has nothing to
do), and their plain definitions against differences."""
import ctypes as C
import math

import numpy as np
import pytest
import torch
import torch.autograd.forward_ad as fwd

import paper_2203_14883_amd as P
from oracle import layer as O
from paper_2203_14883_amd import binding as B
from paper_2203_14883_amd import layer

FAKE = 0x10000  # never dereferenced


def _group(**kw):
    a = dict(types=FAKE, wide=0, num_ids=9, ids=None, n=20_000, G=5, order=FAKE, offsets=FAKE, ws=FAKE, bytes=1 << 40)
    a.update(kw)
    return P.lib().tgl_group_rows(a["types"], a["wide"], a["num_ids"], a["ids"], a["n"], a["G"], a["order"], a["offsets"],
                                  a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(n=1 << 31), dict(G=0), dict(G=1025), dict(wide=2), dict(types=None), dict(types=FAKE + 2),
    dict(types=FAKE + 4, wide=1), dict(ids=FAKE + 2), dict(ids=FAKE, num_ids=-1), dict(ids=FAKE, types=None), dict(order=None),
    dict(order=FAKE + 1), dict(offsets=None), dict(offsets=FAKE + 4), dict(ws=FAKE + 4),
])
def test_group_rows_refuses(kw):
    assert _group(**kw) == B.EINVAL


def test_group_rows_workspace():
    need = P.lib().tgl_group_rows_workspace
    assert need(0, 5) == need(1000, 5) == 0 and need(1_000_000, 5) > 0
    assert need(-1, 5) == need(1 << 31, 5) == need(10, 0) == need(10, 1025) == 0
    assert _group(ws=None) == B.ENOSPACE and _group(bytes=need(20_000, 5) - 1) == B.ENOSPACE
    assert need((1 << 31) - 1, 1024) < 2 ** 33            # 2 bytes a row, counts of at most 8192 chunks


def _groups(**kw):
    a = dict(order=FAKE, offsets=FAKE, n=100, G=4, reserved=0)
    a.update(kw)
    return B.c_row_groups(a["order"], a["offsets"], a["n"], a["G"], a["reserved"])


def _weights(**kw):
    a = dict(ptr=FAKE, ts=32 * 64, rs=64, out=32, in_=64)
    a.update(kw)
    return B.c_typed_weights(a["ptr"], a["ts"], a["rs"], a["out"], a["in_"])


BAD_GROUPS = [dict(offsets=None), dict(offsets=FAKE + 4), dict(order=FAKE + 2), dict(n=-1), dict(n=1 << 31), dict(G=0), dict(G=1025),
              dict(reserved=1)]
BAD_WEIGHTS = [dict(ptr=None), dict(ptr=FAKE + 1), dict(rs=63), dict(out=0), dict(in_=0), dict(out=65537), dict(in_=65537, rs=65537)]


def _linear(groups=None, weights=None, **kw):
    a = dict(x=FAKE, xs=64, bias=None, y=FAKE, ys=32, dt=0)
    a.update(kw)
    return P.lib().tgl_linear_typed(C.byref(groups or _groups()), a["x"], a["xs"], C.byref(weights or _weights()), a["bias"], a["y"],
                                    a["ys"], a["dt"], None)


def _grad_x(groups=None, weights=None, **kw):
    a = dict(x=FAKE, xs=32, y=FAKE, ys=64, dt=0)
    a.update(kw)
    return P.lib().tgl_linear_typed_grad_x(C.byref(groups or _groups()), a["x"], a["xs"], C.byref(weights or _weights()), a["y"],
                                           a["ys"], a["dt"], None)


@pytest.mark.parametrize("call", [_linear, _grad_x])
def test_products_refuse(call):
    for kw in BAD_GROUPS:
        assert call(groups=_groups(**kw)) == B.EINVAL, kw
    for kw in BAD_WEIGHTS:
        assert call(weights=_weights(**kw)) == B.EINVAL, kw
    for kw in [dict(x=None), dict(y=None), dict(x=FAKE + 2), dict(y=FAKE + 1, dt=1), dict(dt=2), dict(ys=31)]:
        assert call(**kw) == B.EINVAL, kw
    assert _linear(bias=FAKE + 2) == B.EINVAL
    assert call(groups=_groups(n=0, order=None), x=None, y=None) == 0


def _grad_w(groups=None, **kw):
    a = dict(dy=FAKE, dys=32, x=FAKE, xs=64, out=32, in_=64, dw=FAKE, db=None, dt=0, ws=FAKE, bytes=1 << 50)
    a.update(kw)
    return P.lib().tgl_linear_typed_grad_w(C.byref(groups or _groups()), a["dy"], a["dys"], a["x"], a["xs"], a["out"], a["in_"],
                                           a["dw"], a["db"], a["dt"], a["ws"], a["bytes"], None)


def test_weights_gradient_refuses():
    for kw in BAD_GROUPS:
        assert _grad_w(groups=_groups(**kw)) == B.EINVAL, kw
    for kw in [dict(dy=None), dict(x=None), dict(dw=None), dict(dy=FAKE + 2), dict(x=FAKE + 1, dt=1), dict(dw=FAKE + 2), dict(db=FAKE + 2),
               dict(out=0), dict(in_=0), dict(out=65537), dict(in_=65537), dict(dt=3)]:
        assert _grad_w(**kw) == B.EINVAL, kw
    many = _groups(n=1_000_000)
    need = P.lib().tgl_linear_typed_grad_w_workspace(C.byref(many), 32, 64, 0)
    assert need > 0
    assert _grad_w(groups=many, bytes=need - 1) == B.ENOSPACE and _grad_w(groups=many, ws=None) == B.ENOSPACE
    assert _grad_w(groups=many, ws=FAKE + 4) == B.EINVAL
    # parts are kept of types that are cut into several only, whatever the number of types
    some = _groups(n=130_000, G=300)
    assert P.lib().tgl_linear_typed_grad_w_workspace(C.byref(some), 4096, 1024, 0) < 12 * 4096 * 1024 * 4


def _norm(**kw):
    a = dict(x=FAKE, xs=64, r=None, rs=0, w=None, b=None, n=3, dim=64, dt=0, eps=1e-5, y=FAKE, ys=64, sum=None, ss=64, stats=None)
    a.update(kw)
    return P.lib().tgl_layer_norm(a["x"], a["xs"], a["r"], a["rs"], a["w"], a["b"], a["n"], a["dim"], a["dt"], a["eps"], a["y"],
                                  a["ys"], a["sum"], a["ss"], a["stats"], None)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(dim=0), dict(dim=16385), dict(dt=2), dict(eps=-1.0), dict(eps=math.nan), dict(x=None), dict(y=None),
    dict(r=FAKE), dict(sum=FAKE), dict(x=FAKE + 2), dict(x=FAKE + 1, dt=1), dict(r=FAKE + 1, sum=FAKE), dict(w=FAKE + 2),
    dict(b=FAKE + 2), dict(y=FAKE + 2), dict(ys=63), dict(r=FAKE, sum=FAKE, ss=63), dict(stats=FAKE + 4),
])
def test_layer_norm_refuses(kw):
    assert _norm(**kw) == B.EINVAL
    assert _norm(n=0, x=None, y=None) == 0


def _norm_grad(**kw):
    a = dict(dy=FAKE, dys=64, h=FAKE, hs=64, stats=FAKE, w=None, dh=None, dhs=0, n=3, dim=64, dt=0, dx=FAKE, dxs=64, dw=FAKE, db=FAKE,
             ws=FAKE, bytes=1 << 40)
    a.update(kw)
    return P.lib().tgl_layer_norm_grad(a["dy"], a["dys"], a["h"], a["hs"], a["stats"], a["w"], a["dh"], a["dhs"], a["n"], a["dim"],
                                       a["dt"], a["dx"], a["dxs"], a["dw"], a["db"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(dim=0), dict(dim=16385), dict(dt=2), dict(dy=None), dict(h=None), dict(stats=None), dict(dy=FAKE + 2),
    dict(h=FAKE + 1, dt=1), dict(dh=FAKE + 2), dict(dx=FAKE + 2), dict(dxs=63), dict(w=FAKE + 2), dict(stats=FAKE + 4),
    dict(dw=FAKE + 2), dict(db=FAKE + 2), dict(ws=FAKE + 4),
])
def test_layer_norm_grad_refuses(kw):
    assert _norm_grad(**kw) == B.EINVAL


def test_layer_norm_grad_workspace():
    need = P.lib().tgl_layer_norm_grad_workspace(3, 64)
    assert need > 0 and _norm_grad(bytes=need - 1) == B.ENOSPACE and _norm_grad(ws=None) == B.ENOSPACE
    assert _norm_grad(dx=None, dw=None, db=None, ws=None) == 0
    assert P.lib().tgl_layer_norm_grad_workspace(-1, 64) == P.lib().tgl_layer_norm_grad_workspace(3, 16385) == 0


def _all(x, w, g, t):
    stats = torch.zeros(len(x), 2, dtype=torch.float64)
    return (lambda: P.group_rows(t, 3), lambda: P.linear_typed(x, w, g), lambda: P.linear_typed_backward(x, x, w, g),
            lambda: P.layer_norm(x), lambda: P.layer_norm_backward(x, x, stats))


def test_python_refuses_host_tensors_and_tangents():
    x, w = torch.randn(4, 32), torch.randn(3, 32, 32)
    t = torch.zeros(4, dtype=torch.int32)
    g = P.RowGroups(torch.zeros(4, dtype=torch.int64), t)
    for f in _all(x, w, g, t):
        with pytest.raises(ValueError, match="current device"):
            f()
    with fwd.dual_level():
        dual = fwd.make_dual(x, torch.ones_like(x))
        with pytest.raises(ValueError, match="tangent"):
            layer._also(dual, "x", -1)
        layer._also(x, "x", -1)
        layer._also(fwd.unpack_dual(dual).primal, "x", -1)


@pytest.mark.parametrize("offsets,order", [
    (torch.zeros(4, dtype=torch.int32), None), (torch.zeros(1, dtype=torch.int64), None), (torch.zeros(1026, dtype=torch.int64), None),
    (torch.zeros(4, 2, dtype=torch.int64), None), (torch.zeros(8, dtype=torch.int64)[::2], None),
    (torch.zeros(4, dtype=torch.int64), torch.zeros(9, dtype=torch.int64)),
    (torch.zeros(4, dtype=torch.int64), torch.zeros(18, dtype=torch.int32)[::2]),
])
def test_row_groups_refuse(offsets, order):
    with pytest.raises(ValueError):
        P.RowGroups(offsets, order)


def test_row_groups_of_other_rows_are_refused():
    g = P.RowGroups(torch.zeros(4, dtype=torch.int64), torch.zeros(9, dtype=torch.int32))
    assert g.num_types == 3 and g.c_view(9, -1).n == 9
    with pytest.raises(ValueError, match="9 rows"):
        g.c_view(8, -1)
    assert P.RowGroups(g.offsets).c_view(8, -1).order is None


def test_weights_of_other_shapes_are_refused():
    g = P.RowGroups(torch.zeros(4, dtype=torch.int64))
    f32 = torch.float32
    good = torch.zeros(3, 5, 7)
    v = layer._weights(good, g, f32, -1)
    assert (v.type_stride, v.row_stride, v.out, v.in_) == (35, 7, 5, 7)
    v = layer._weights(good[:1].expand(3, 5, 7), g, f32, -1)            # one matrix for all types
    assert (v.type_stride, v.row_stride) == (0, 7)
    v = layer._weights(torch.zeros(3, 5, 16)[:, :, 2:9], g, f32, -1)
    assert (v.type_stride, v.row_stride, v.in_) == (80, 16, 7)
    for bad in (good[:2], good[0], good.double(), good.to(torch.bfloat16), good.transpose(1, 2), good[:, :1].expand(3, 5, 7),
                torch.zeros(3, 0, 7), torch.zeros(3, 7, 0)):
        with pytest.raises(ValueError):
            layer._weights(bad, g, f32, -1)


def test_gradients_are_not_recorded_under_capture(monkeypatch):
    """Refused before anything is enqueued; without a gradient the call goes on to its other checks."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    monkeypatch.setattr(layer, "_device", lambda t, name: -1)
    x, w = torch.randn(4, 32, requires_grad=True), torch.randn(2, 32, 32)
    g = P.RowGroups(torch.zeros(4, dtype=torch.int64))
    for f in (lambda t: P.linear_typed(t, w, g), lambda t: P.layer_norm(t, w)):
        with pytest.raises(RuntimeError, match="captured"):
            f(x)
        with pytest.raises(ValueError, match="w must be|weight must be"):
            f(x.detach())
    for f, rest in ((layer._LinearTyped, ()), (layer._LayerNorm, (None,))):
        with pytest.raises(RuntimeError, match="captured"):
            f.backward(None, x.detach(), *rest)


def test_out_has_no_gradient():
    x, w = torch.randn(4, 32, requires_grad=True), torch.randn(3, 32, 32)
    with pytest.raises(ValueError, match="out"):
        P.linear_typed(x, w, P.RowGroups(torch.zeros(4, dtype=torch.int64)), out=torch.zeros(4, 32))


def test_oracle_of_a_hand_written_call():
    order, offsets, t = O.group_rows([2, 0, 5, 2, -1], 3)
    assert order.tolist() == [1, 0, 3, 2, 4] and offsets.tolist() == [0, 1, 1, 3] and t.tolist() == [2, 0, -1, 2, -1]
    order, offsets, t = O.group_rows([1, 0], 2, ids=[0, -1, 1, 7, 0])
    assert t.tolist() == [1, -1, 0, -1, 1] and order.tolist() == [2, 0, 4, 1, 3]
    w = np.array([[[1.0, 2.0]], [[3.0, 4.0]]])
    y = O.linear(np.array([[1.0, 1.0], [2.0, 0.0], [5.0, 5.0]]), w, np.array([1, 0, -1]), np.array([[10.0], [20.0]]))
    assert y.tolist() == [[27.0], [12.0], [0.0]]


def test_oracle_gradients_are_differences():
    rng = np.random.default_rng(3)
    t = np.array([0, 2, -1, 2, 0])
    x, w, d = rng.standard_normal((5, 4)), rng.standard_normal((3, 6, 4)), rng.standard_normal((5, 6))
    dx, dw, db = O.linear_backward(d, x, w, t)
    gamma, beta = rng.standard_normal(4), rng.standard_normal(4)
    dn = rng.standard_normal((5, 4))
    nx, ng, nb = O.layer_norm_backward(dn, x, gamma)

    def slope(f, a, i, step=1e-5):
        keep = a[i]
        a[i] = keep + step
        hi = f()
        a[i] = keep - step
        lo = f()
        a[i] = keep
        return (hi - lo) / (2 * step)

    linear = lambda: (O.linear(x, w, t, b) * d).sum()
    norm = lambda: (O.layer_norm(x, gamma, beta)[0] * dn).sum()
    b = rng.standard_normal((3, 6))
    for f, a, got in ((linear, x, dx), (linear, w, dw), (linear, b, db), (norm, x, nx), (norm, gamma, ng), (norm, beta, nb)):
        for i in np.ndindex(a.shape):
            # central differences: the third derivative's term (of order 1e-10 here) and 1e-16 / 1e-5 of rounding
            assert abs(slope(f, a, i) - got[i]) < 1e-7
