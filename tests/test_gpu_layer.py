"""The training operators against their plain definitions in 64 bits (oracle/layer.py)."""
import math

import numpy as np
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu
from oracle import layer as O

pytestmark = pytest.mark.gpu
DTYPES = ["f32", "bf16"]
UNIT = 2.0 ** -23       # a unit in the last place of a float32 near 1
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}     # half a step of the result's type, beyond float32's


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


def _type(torch, t):
    return torch.float32 if t == "f32" else torch.bfloat16


def _up(torch, a, t="f32"):
    """Device tensor of type t, and its values as the host sees them."""
    x = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(_type(torch, t))
    return x.cuda(), x.double().numpy()


def _host(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, terms, size, dtype):
    """A float32 sum of `terms` products: each product and each addition is off by at most a unit (the matrix
    instructions need not round to nearest) of the products' sizes together, `size`; one rounding to the result's type
    (its half step of what was rounded, so of the value and of that error)."""
    tol = (2 * terms + 8) * UNIT * size
    tol = tol + ROUND[dtype] * (np.abs(want) + tol) + 1e-37
    bad = ~(np.abs(_host(got) - want) <= tol)
    assert not bad.any(), "%d of %d off, first at %s" % (bad.sum(), bad.size, np.argwhere(bad)[0])


# ---- rows by type -----------------------------------------------------------

def _check_groups(torch, types, G, ids=None, dtype=None):
    t = torch.from_numpy(np.asarray(types, np.int64)).to(dtype or torch.int32).cuda()
    i = None if ids is None else torch.from_numpy(np.asarray(ids, np.int32)).cuda()
    g = P.group_rows(t, G, ids=i)
    order, offsets, _ = O.group_rows(types, G, ids)
    assert g.num_types == G and g.order.dtype == torch.int32 and g.offsets.dtype == torch.int64
    assert np.array_equal(g.offsets.cpu().numpy(), offsets)
    assert np.array_equal(g.order.cpu().numpy(), order)


@pytest.mark.parametrize("n,G", [(0, 3), (1, 1), (1, 1024), (63, 2), (64, 64), (65, 63), (1800, 3), (2048, 1024), (2049, 5), (16384, 1000),
                                 (16385, 7), (20_011, 1024), (100_003, 1), (300_000, 300), (1_000_003, 65)])
def test_group_rows(torch, n, G):
    announce("group_rows %d of %d types" % (n, G))
    rng = np.random.default_rng(n + G)
    _check_groups(torch, rng.integers(0, G, n), G)
    _check_groups(torch, rng.integers(-2, G + 3, n), G, dtype=torch.int64)       # some of no type


@pytest.mark.parametrize("n", [5, 3000, 40_000])
def test_group_rows_by_id(torch, n):
    announce("group_rows of %d ids" % n)
    rng = np.random.default_rng(n)
    types = rng.integers(-1, 9, 1000)
    _check_groups(torch, types, 8, rng.integers(-3, 1005, n))
    _check_groups(torch, types, 8, rng.integers(-3, 1005, n), torch.int64)
    _check_groups(torch, types[:0], 8, rng.integers(-3, 5, n))                  # no node has a type
    _check_groups(torch, types, 8, np.full(n, -1))


def test_group_rows_types_beyond_32_bits(torch):
    announce("group_rows wide types")
    wide = np.array([0, 2 ** 32, 2 ** 32 + 1, -2 ** 32, 1, 2 ** 63 - 1, -2 ** 63, 1], np.int64)
    _check_groups(torch, wide, 3, dtype=torch.int64)
    _check_groups(torch, np.tile(wide, 4000), 3, dtype=torch.int64)


@pytest.mark.parametrize("n", [2000, 50_000])
def test_group_rows_all_of_one_type(torch, n):
    announce("group_rows of one type")
    for g in (0, 4, 9, 10):
        _check_groups(torch, np.full(n, g), 10)


# ---- products ---------------------------------------------------------------

SIZES = [
    # rows, in, out, types: one of everything, odd ones, ends of tiles and past them
    (1, 1, 1, 1), (1, 768, 257, 4), (2, 7, 3, 5), (5, 64, 64, 1), (17, 33, 65, 3), (64, 128, 16, 2), (65, 100, 272, 4), (100, 272, 100, 200),
    (129, 31, 130, 2), (130, 513, 40, 3), (300, 72, 129, 7), (257, 256, 256, 1), (700, 264, 136, 3), (1000, 65, 1000, 5), (40, 1040, 520, 2),
]


def _case(rng, n, k, out, G, empty=0.1):
    t = rng.integers(0, G, n)
    t[rng.random(n) < empty] = -1
    if n > 20 and G > 2:
        t[t == 1] = 0                       # a type without rows
    return t


def _check_linear(torch, dtype, t, G, x, w, b, d, groups=None, x_host=None, w_host=None, d_host=None):
    """x, w, d on the device; all four results against the definition."""
    g = groups if groups is not None else P.group_rows(torch.from_numpy(np.asarray(t, np.int32)).cuda(), G)
    xh, wh, dh = (_host(v) for v in (x, w, d))
    bh = None if b is None else _host(b)
    k, out, n = x.shape[1], w.shape[1], len(xh)
    y = P.linear_typed(x, w, g, b)
    dx, dw, db = P.linear_typed_backward(d, x, w, g, bias=True)
    assert y.dtype == dx.dtype == dw.dtype == x.dtype and db.dtype == torch.float32
    assert y.shape == (n, out) and dx.shape == x.shape and dw.shape == (G, out, k) and db.shape == (G, out)
    _close(y, O.linear(xh, wh, t, bh), k + 1, O.linear(np.abs(xh), np.abs(wh), t, None if b is None else np.abs(bh)), dtype)
    wx, ww, wb = O.linear_backward(dh, xh, wh, t)
    sx, sw, sb = O.linear_backward(np.abs(dh), np.abs(xh), np.abs(wh), t)
    most = max([1] + [int((t == g).sum()) for g in range(G)])
    _close(dx, wx, out, sx, dtype)
    _close(dw, ww, most, sw, dtype)
    _close(db, wb, most, sb, "f32")
    none = np.flatnonzero(np.asarray(t) < 0)
    assert not _host(y)[none].any() and not _host(dx)[none].any()
    return y, dx, dw, db


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k,out,G", SIZES)
def test_linear_typed(torch, n, k, out, G, dtype):
    announce("linear_typed %d x %d -> %d, %d types, %s" % (n, k, out, G, dtype))
    rng = np.random.default_rng(n * 7 + k * 3 + out + G)
    t = _case(rng, n, k, out, G)
    x, _ = _up(torch, rng.standard_normal((n, k)), dtype)
    w, _ = _up(torch, rng.standard_normal((G, out, k)), dtype)
    d, _ = _up(torch, rng.standard_normal((n, out)), dtype)
    b, _ = _up(torch, rng.standard_normal((G, out)))
    _check_linear(torch, dtype, t, G, x, w, b, d)
    _check_linear(torch, dtype, t, G, x, w, None, d)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k,out,G,empty", [(5000, 272, 100, 3, 0.1), (5003, 100, 272, 2, 0.0), (20_000, 64, 72, 40, 0.3), (3001, 520, 776, 2, 0.0),
                                             (9000, 128, 256, 1, 0.0), (4096, 768, 1024, 3, 0.05), (2500, 1023, 515, 2, 0.1), (1500, 1024, 2304, 1, 0.0),
                                             (70_000, 48, 33, 3, 0.9), (40_000, 200, 264, 200, 0.0), (50_000, 256, 512, 6, 0.02),
                                             (42_000, 264, 328, 3, 0.1), (33_000, 67, 45, 2, 0.0), (60, 2000, 1030, 3, 0.1)])
def test_linear_typed_of_many_rows(torch, n, k, out, G, empty, dtype):
    """Sums over rows in several parts, tiles of every size."""
    announce("linear_typed of many %d x %d -> %d, %d types, %s" % (n, k, out, G, dtype))
    rng = np.random.default_rng(n + k + out)
    t = np.minimum(rng.geometric(0.5, n) - 1, G - 1)        # some types have many rows, others few or none
    t = (t * 37 + 3) % G
    t[rng.random(n) < empty] = -1
    x, _ = _up(torch, rng.standard_normal((n, k)), dtype)
    w, _ = _up(torch, rng.standard_normal((G, out, k)), dtype)
    d, _ = _up(torch, rng.standard_normal((n, out)), dtype)
    b, _ = _up(torch, rng.standard_normal((G, out)))
    g = P.group_rows(torch.from_numpy(t.astype(np.int32)).cuda(), G)
    xh, wh, dh, bh = (_host(v) for v in (x, w, d, b))
    y = P.linear_typed(x, w, g, b)
    dx, dw, db = P.linear_typed_backward(d, x, w, g, bias=True)
    # by matrix products on the host, type by type
    want, size = np.zeros((n, out)), np.zeros((n, out))
    for i in range(G):
        r = t == i
        want[r], size[r] = xh[r] @ wh[i].T + bh[i], np.abs(xh[r]) @ np.abs(wh[i]).T + np.abs(bh[i])
    _close(y, want, k + 1, size, dtype)
    wx, ww, wb = O.linear_backward(dh, xh, wh, t)
    sx, sw, sb = O.linear_backward(np.abs(dh), np.abs(xh), np.abs(wh), t)
    _close(dx, wx, out, sx, dtype)
    _close(dw, ww, n, sw, dtype)
    _close(db, wb, n, sb, "f32")
    again = P.linear_typed_backward(d, x, w, g, bias=True)
    for a, c in zip((dx, dw, db), again):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_typed_rows_in_order(torch, dtype):
    """Without an order: rows lie in their types' order, those behind the last type's have none."""
    announce("linear_typed in order")
    rng = np.random.default_rng(5)
    offsets = np.array([0, 3, 3, 140, 200])
    t = np.full(230, -1)
    for g in range(4):
        t[offsets[g]:offsets[g + 1]] = g
    x, w, d = (_up(torch, rng.standard_normal(s), dtype)[0] for s in ((230, 72), (4, 96, 72), (230, 96)))
    g = P.RowGroups(torch.from_numpy(offsets).cuda())
    _check_linear(torch, dtype, t, 4, x, w, None, d, groups=g)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k,out", [(64, 48), (67, 45)])
def test_linear_typed_strides(torch, k, out, dtype):
    """Slices of wider tensors, rows broadcast, weights broadcast over types, an output between other columns."""
    announce("linear_typed strides %d %d" % (k, out))
    rng = np.random.default_rng(k)
    n, G = 150, 3
    t = _case(rng, n, k, out, G)
    x = _up(torch, rng.standard_normal((n, 2 * k + 3)), dtype)[0][:, 3:3 + k]
    d = _up(torch, rng.standard_normal((2 * n, out + 5)), dtype)[0][::2, 1:1 + out]
    w = _up(torch, rng.standard_normal((G, out + 2, k + 9)), dtype)[0][:, 1:1 + out, 4:4 + k]
    _check_linear(torch, dtype, t, G, x, w, None, d)
    _check_linear(torch, dtype, t, G, x[:1].expand(n, k), w[1:2].expand(G, out, k), None, d)
    g = P.group_rows(torch.from_numpy(t.astype(np.int32)).cuda(), G)
    wide = torch.full((n + 2, out + 7), 7.0, device="cuda", dtype=x.dtype)
    into = wide[1:-1, 3:3 + out]
    assert P.linear_typed(x, w, g, out=into) is into
    assert torch.equal(into, P.linear_typed(x, w, g))
    into.fill_(7.0)
    assert torch.equal(wide, torch.full_like(wide, 7.0))


def test_linear_typed_of_nothing(torch):
    announce("linear_typed of nothing")
    g = P.group_rows(torch.zeros(0, dtype=torch.int32, device="cuda"), 3)
    x, w = torch.zeros(0, 8, device="cuda"), torch.ones(3, 5, 8, device="cuda")
    assert P.linear_typed(x, w, g).shape == (0, 5)
    dx, dw, db = P.linear_typed_backward(torch.zeros(0, 5, device="cuda"), x, w, g, bias=True)
    assert dx.shape == (0, 8) and not dw.any() and not db.any()
    g = P.group_rows(torch.full((70,), -1, dtype=torch.int32, device="cuda"), 3)
    x = torch.full((70, 8), math.nan, device="cuda")               # rows of no type are not read
    assert not P.linear_typed(x, w, g, torch.ones(3, 5, device="cuda")).any()
    dx, dw, db = P.linear_typed_backward(torch.full((70, 5), math.nan, device="cuda"), x, w, g, bias=True)
    assert not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_typed_keeps_rows_apart(torch, dtype):
    """Rows of NaN and infinity change their own results, their type's gradients, and nothing else."""
    announce("linear_typed with NaN")
    rng = np.random.default_rng(11)
    n, k, out, G = 200, 40, 72, 4
    t = rng.integers(0, 3, n)
    t[5], t[6], t[7] = 3, 3, -1
    x, w, d = (_up(torch, rng.standard_normal(s), dtype)[0] for s in ((n, k), (G, out, k), (n, out)))
    g = P.group_rows(torch.from_numpy(t.astype(np.int32)).cuda(), G)
    y0, (dx0, dw0, db0) = P.linear_typed(x, w, g), P.linear_typed_backward(d, x, w, g, bias=True)
    for v in (x, d):
        v[5], v[6], v[7] = math.nan, math.inf, math.nan
    w[3] = math.nan
    y1, (dx1, dw1, db1) = P.linear_typed(x, w, g), P.linear_typed_backward(d, x, w, g, bias=True)
    others = torch.from_numpy(t < 3).cuda()
    assert torch.equal(y0[others], y1[others]) and torch.equal(dx0[others], dx1[others])
    assert torch.equal(dw0[:3], dw1[:3]) and torch.equal(db0[:3], db1[:3])
    assert torch.isnan(y1[5]).all() and torch.isnan(dw1[3]).all() and torch.isnan(db1[3]).all() and not y1[7].any()


def test_groups_that_make_no_sense_stay_within_the_rows(torch):
    """Offsets and places beyond the rows: nothing is read or written outside, other rows are as they were."""
    announce("groups that make no sense")
    n, k, out, G = 100, 64, 64, 3
    x, w = torch.randn(n, k, device="cuda"), torch.randn(G, out, k, device="cuda")
    order = torch.arange(n, dtype=torch.int32, device="cuda")
    order[::7] = 10 ** 9
    order[3::7] = -5
    for offsets in ([0, 40, 80, 10 ** 12], [0, -7, 50, 90], [0, 90, 20, 100], [5, 300, 400, 500]):
        g = P.RowGroups(torch.tensor(offsets, dtype=torch.int64, device="cuda"), order)
        wide = torch.full((n + 2, out), 3.0, device="cuda")
        P.linear_typed(x, w, g, out=wide[1:-1])
        assert bool((wide[0] == 3).all()) and bool((wide[-1] == 3).all())
        assert bool((wide[1:-1][torch.cat([torch.arange(0, n, 7), torch.arange(3, n, 7)]).cuda()] == 3).all())
        P.linear_typed_backward(x, x, w, g, bias=True)
        torch.cuda.synchronize()


# ---- layer norm -------------------------------------------------------------

DIMS = [1, 2, 7, 8, 31, 64, 65, 100, 128, 129, 172, 256, 257, 512, 513, 768, 1000, 1024, 1025, 2048, 2049, 4096, 4101, 8192, 8200, 16384]


def _norm_case(torch, rng, n, dim, dtype, residual, params):
    x, _ = _up(torch, 3 * rng.standard_normal((n, dim)) + rng.standard_normal((n, 1)), dtype)
    r = _up(torch, rng.standard_normal((n, dim)), dtype)[0] if residual else None
    w = _up(torch, 1 + 0.2 * rng.standard_normal(dim))[0] if params else None
    b = _up(torch, 0.2 * rng.standard_normal(dim))[0] if params else None
    return x, r, w, b


def _check_norm(torch, dtype, x, r, w, b, d, dh, eps=1e-5):
    got = P.layer_norm(x, w, b, residual=r, eps=eps, return_stats=True)
    y, stats = got[0], got[-1]
    if r is None:
        assert len(got) == 2
        h = x
    else:
        h = got[1]
        # the sum of two numbers in float32, rounded to their type
        assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    hh, wh, bh, dyh = _host(h), None if w is None else _host(w), None if b is None else _host(b), _host(d)
    want, mean, rstd, xh = O.layer_norm(hh, wh, bh, np.float64(np.float32(eps)))
    dim = hh.shape[1]
    # sums of 64 bits: rounding of the operands aside, which a mean that is large beside the distances magnifies
    np.testing.assert_allclose(_host(stats)[:, 0], mean, rtol=0, atol=dim * 2.0 ** -53 * max(1e-300, np.abs(hh).max()))
    np.testing.assert_allclose(_host(stats)[:, 1], rstd, rtol=dim * 2.0 ** -48)
    # (h - mean) rstd to float32, a product and a sum: a half unit each of what they give, then the result's type
    parts = np.abs(xh * (1 if wh is None else wh)) + np.abs(want)
    tol = UNIT * parts
    assert (np.abs(_host(y) - want) <= tol + ROUND[dtype] * (np.abs(want) + tol) + 1e-37).all()
    dx, dw, db = P.layer_norm_backward(d, h, stats, w, dh=dh)
    wx, ww, wb = O.layer_norm_backward(dyh, hh, wh, np.float64(np.float32(eps)))
    if dh is not None:
        wx = wx + _host(dh)
    # In half units of float32: xh = ((h - upper) - lower) rstd is off by 4 (three operations, rstd), g = dy w by 1.  The
    # means' sums are of 32 bits over a lane's elements, 32 at most, and of 64 over the lanes: mean(g) is off by 1 + 32 and
    # mean(g xh) by 1 + 4 + 32 of what they add up, and by 1 when they are rounded.  g - mean(g), the product with xh (4 off),
    # the difference, the product with rstd (1 off) and dh's addition: 1 each of what goes into them.
    g = np.abs(dyh * (1 if wh is None else wh))
    size = (40 * g.mean(1, keepdims=True) + 6 * g + 48 * np.abs(xh) * (g * np.abs(xh)).mean(1, keepdims=True)) * rstd[:, None]
    tol = UNIT / 2 * (size + 2 * np.abs(wx))
    assert (np.abs(_host(dx) - wx) <= tol + ROUND[dtype] * (np.abs(wx) + tol) + 1e-37).all()
    # 4 of xh, 1 a row for at most 32 rows in 32 bits, the result's own
    assert (np.abs(_host(dw) - ww) <= UNIT / 2 * 38 * np.abs(dyh * xh).sum(0) + 1e-37).all()
    assert (np.abs(_host(db) - wb) <= UNIT / 2 * 34 * np.abs(dyh).sum(0) + 1e-37).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_layer_norm(torch, dim, dtype):
    rng = np.random.default_rng(dim)
    for n, residual, params in ((1, False, True), (5, True, True), (67, True, False), (3, False, False)):
        announce("layer_norm %d x %d %s" % (n, dim, dtype))
        x, r, w, b = _norm_case(torch, rng, n, dim, dtype, residual, params)
        d = _up(torch, rng.standard_normal((n, dim)), dtype)[0]
        dh = _up(torch, rng.standard_normal((n, dim)), dtype)[0] if residual else None
        _check_norm(torch, dtype, x, r, w, b, d, dh)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,dim", [(40_000, 16), (12_001, 100), (9001, 200), (9000, 768), (5000, 1500), (2600, 2100), (1300, 4100), (140_000, 132),
                                   (17_000, 2052), (8400, 4101)])
def test_layer_norm_of_many_rows(torch, n, dim, dtype):
    """More rows than one turn of every workgroup takes, and more than a lane sums in 32 bits."""
    announce("layer_norm of many %d x %d %s" % (n, dim, dtype))
    rng = np.random.default_rng(n)
    x, r, w, b = _norm_case(torch, rng, n, dim, dtype, True, True)
    d, dh = (_up(torch, rng.standard_normal((n, dim)), dtype)[0] for _ in range(2))
    _check_norm(torch, dtype, x, r, w, b, d, dh)


@pytest.mark.parametrize("dtype", DTYPES)
def test_layer_norm_strides(torch, dtype):
    announce("layer_norm strides")
    rng = np.random.default_rng(2)
    wide = _up(torch, rng.standard_normal((40, 3 * 131 + 2)), dtype)[0]
    x, r, d = wide[:, 1:132], wide[::1, 132:263], wide[:, 263:394]
    _check_norm(torch, dtype, x, r, None, None, d, None)
    _check_norm(torch, dtype, x[3:4].expand(40, 131), r, None, None, d[1:2].expand(40, 131), x)


def test_layer_norm_of_extremes(torch):
    """A large mean beside small distances, rows of the largest and the smallest numbers, rows of one number."""
    announce("layer_norm of extremes")
    rng = np.random.default_rng(4)
    h = rng.standard_normal((9, 300))
    h[0] = 1e4 + 1e-2 * h[0]
    h[1] *= 1e37
    h[2] = np.where(h[2] > 0, 3.4e38, -3.4e38)
    h[3] = 3.4e38
    h[4] *= 1e-37
    h[5] = 0.0
    h[6] = 1e30
    h[7] = 5.0
    h[7, 0] = 5.0 + 2.0 ** -20
    x = torch.from_numpy(h.astype(np.float32)).cuda()
    d = torch.from_numpy(rng.standard_normal((9, 300)).astype(np.float32)).cuda()
    _check_norm(torch, "f32", x, None, None, None, d, None)
    _check_norm(torch, "f32", x[:3], None, None, None, d[:3], None, eps=0.0)


def test_layer_norm_of_what_is_no_number(torch):
    announce("layer_norm of NaN")
    x = torch.randn(6, 50, device="cuda")
    y0 = P.layer_norm(x)
    x[2, 7], x[4, 49] = math.nan, math.inf
    y = P.layer_norm(x)
    assert torch.isnan(y[2]).all() and torch.isnan(y[4]).all()
    rest = torch.tensor([0, 1, 3, 5], device="cuda")
    assert torch.equal(y[rest], y0[rest])


def test_layer_norm_of_nothing(torch):
    announce("layer_norm of nothing")
    x = torch.zeros(0, 50, device="cuda")
    y, h, stats = P.layer_norm(x, residual=x, return_stats=True)
    assert y.shape == h.shape == (0, 50) and stats.shape == (0, 2)
    dx, dw, db = P.layer_norm_backward(x, h, stats)
    assert dx.shape == (0, 50) and not dw.any() and not db.any()


# ---- gradients as torch records them ----------------------------------------

def test_recorded_gradients_are_the_calls(torch):
    """A layer's step through autograd: the same bits as the calls of their own, leaves of every kind."""
    announce("recorded gradients")
    n, k, out, G = 500, 72, 104, 3
    t = torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32)
    g = P.group_rows(t, G)
    for dtype in (torch.float32, torch.bfloat16):
        x, w, r = (torch.randn(*s, device="cuda").to(dtype).requires_grad_() for s in ((n, k), (G, out, k), (n, out)))
        b, gamma, beta = (torch.randn(*s, device="cuda").requires_grad_() for s in ((G, out), (out,), (out,)))
        d, dh = torch.randn(n, out, device="cuda").to(dtype), torch.randn(n, out, device="cuda").to(dtype)
        y, h = P.layer_norm(P.linear_typed(x, w, g, b), gamma, beta, residual=r)
        got = torch.autograd.grad((y, h), (x, w, b, gamma, beta, r), (d, dh))
        with torch.no_grad():
            z = P.linear_typed(x, w, g, b)
            y2, h2, stats = P.layer_norm(z, gamma, beta, residual=r, return_stats=True)
            dz, dgamma, dbeta = P.layer_norm_backward(d, h2, stats, gamma, dh=dh)
            dx, dw, db = P.linear_typed_backward(dz, x, w, g, bias=True)
        assert torch.equal(y, y2) and torch.equal(h, h2)
        for a, c in zip(got, (dx, dw, db, dgamma, dbeta, dz)):
            assert torch.equal(a, c)
        # one leaf at a time, a gradient that is broadcast, and only the sum used
        for leaf, c in ((x, dx), (w, dw), (b, db)):
            other = [v.detach() for v in (x, w, b)]
            other[[x is leaf, w is leaf, b is leaf].index(True)] = leaf
            y3 = P.linear_typed(other[0], other[1], g, other[2])
            assert torch.equal(torch.autograd.grad(y3, leaf, dz)[0], c)
        y3 = P.linear_typed(x, w, g, b)
        ones = torch.autograd.grad(y3.sum(), x)[0]
        assert torch.equal(ones, P.linear_typed_backward(torch.ones_like(y3), x, w, g)[0])
        _, h = P.layer_norm(x.detach(), None, None, residual=x)
        assert torch.equal(torch.autograd.grad(h, x, x.detach())[0], x)


def test_gradients_against_differences(torch):
    """Central differences of a float32 step: two values of it that are off by a few units of the largest part of
    their sum, over the distance, and the third derivative's term."""
    announce("gradients against differences")
    torch.manual_seed(3)
    n, k, out, G = 12, 9, 10, 3
    t = torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32)
    g = P.group_rows(t, G)
    leaves = [torch.randn(*s, device="cuda").requires_grad_() for s in ((n, k), (G, out, k), (G, out), (out,), (out,), (n, out))]
    d = torch.randn(n, out, device="cuda")

    def value(*v):
        y, h = P.layer_norm(P.linear_typed(v[0], v[1], g, v[2]), v[3], v[4], residual=v[5], eps=0.1)
        return ((y * d).double().sum() + (h * d).double().sum())

    grads = torch.autograd.grad(value(*leaves), leaves)
    with torch.no_grad():
        for i, leaf in enumerate(leaves):
            along = torch.randn_like(leaf)
            step = 2.0 ** -8
            v = [x.clone() for x in leaves]
            v[i] = leaf + step * along
            hi = value(*v)
            v[i] = leaf - step * along
            lo = value(*v)
            slope = float((hi - lo) / (2 * step))
            want = float((grads[i].double() * along.double()).sum())
            # 2 * n * out terms of size up to about 30, each off by up to 16 half units; third derivatives of order 100 here
            noise = 2 * n * out * 30 * 16 * UNIT / 2 / step
            assert abs(slope - want) <= noise + 100 * step ** 2 * float(along.square().sum()), i


def test_operators_run_together_on_a_sampled_batch(torch):
    """Types of sampled slots, their projection, the norm: as a temporal layer uses them."""
    announce("a sampled batch")
    rng = np.random.default_rng(9)
    N, E, G = 300, 4000, 3
    src, dst = (torch.from_numpy(rng.integers(0, N, E).astype(np.int32)).cuda() for _ in range(2))
    ts = torch.arange(E, dtype=torch.float32, device="cuda")
    graph = P.tcsr_build(src, dst, ts, None, N, True)
    roots = torch.from_numpy(rng.integers(0, N, 64).astype(np.int32)).cuda()
    hop = P.sample(graph, roots, torch.full((64,), 2000.0, device="cuda"), fanouts=(10,), mode="recent")[0]
    nbr = hop.nbr.reshape(-1)
    kind = torch.from_numpy(rng.integers(0, G, N).astype(np.int32)).cuda()
    groups = P.group_rows(kind, G, ids=nbr)
    ids = nbr.cpu().numpy()
    t = np.where(ids < 0, -1, kind.cpu().numpy()[np.maximum(ids, 0)])
    order, offsets, _ = O.group_rows(kind.cpu().numpy(), G, ids)
    assert (t < 0).any() and np.array_equal(groups.order.cpu().numpy(), order) and np.array_equal(groups.offsets.cpu().numpy(), offsets)
    x = torch.randn(len(ids), 40, device="cuda")
    w, b, d = torch.randn(G, 24, 40, device="cuda"), torch.randn(G, 24, device="cuda"), torch.randn(len(ids), 24, device="cuda")
    _check_linear(torch, "f32", t, G, x, w, b, d, groups=groups)
    z = P.linear_typed(x, w, groups, b)
    gamma, beta = torch.randn(24, device="cuda"), torch.randn(24, device="cuda")
    _check_norm(torch, "f32", z, d, gamma, beta, x[:, :24], None)


# ---- streams and graphs -----------------------------------------------------

def test_another_stream(torch):
    announce("another stream")
    n, k, out, G = 3000, 64, 96, 3
    t = torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32)
    x, w, d = torch.randn(n, k, device="cuda"), torch.randn(G, out, k, device="cuda"), torch.randn(n, out, device="cuda")
    g = P.group_rows(t, G)
    y = P.linear_typed(x, w, g)
    back = P.linear_typed_backward(d, x, w, g, bias=True)
    z, stats = P.layer_norm(y, return_stats=True)
    nb = P.layer_norm_backward(d, y, stats)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g2 = P.group_rows(t, G, stream=side)
    y2 = P.linear_typed(x, w, g2, stream=side)
    back2 = P.linear_typed_backward(d, x, w, g2, bias=True, stream=side)
    z2, stats2 = P.layer_norm(y2, return_stats=True, stream=side)
    nb2 = P.layer_norm_backward(d, y2, stats2, stream=side)
    with torch.cuda.stream(side):
        xg = x.clone().requires_grad_()
    y3 = P.linear_typed(xg, w, g2, stream=side)
    side.synchronize()
    for a, c in zip((g.order, g.offsets, y, z, *back, *nb, y), (g2.order, g2.offsets, y2, z2, *back2, *nb2, y3)):
        assert torch.equal(a, c)
    with torch.cuda.stream(side):
        dx = torch.autograd.grad(y3, xg, d)[0]
    side.synchronize()
    assert torch.equal(dx, back[0])


def test_captured_step(torch):
    """Two graphs of the same step, replayed with eager work between: every replay is the eager result."""
    announce("captured step")
    n, k, out, G = 20_000, 72, 64, 4
    t = torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32)
    x, w, d = torch.randn(n, k, device="cuda"), torch.randn(G, out, k, device="cuda"), torch.randn(n, out, device="cuda")

    def step():
        g = P.group_rows(t, G)
        y = P.linear_typed(x, w, g)
        z, stats = P.layer_norm(y, return_stats=True)
        dy, dgamma, dbeta = P.layer_norm_backward(d, y, stats)
        return (g.order, g.offsets, y, z, dgamma, dbeta) + P.linear_typed_backward(dy, x, w, g, bias=True)

    step()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step()
        graphs.append((graph, outs))
    for i in range(4):
        t.copy_(torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32))
        x.copy_(torch.randn(n, k, device="cuda"))
        d.copy_(torch.randn(n, out, device="cuda"))
        want = step()
        torch.cuda.synchronize()
        for graph, outs in graphs if i % 2 else graphs[::-1]:
            graph.replay()
            for a, c in zip(outs, want):
                assert torch.equal(a, c)


def test_two_calls_at_once(torch):
    """Two calls at once, on two streams, of the same groups and weights: neither sees the other."""
    announce("two streams at once")
    n, k, out, G = 30_000, 128, 96, 5
    t = torch.randint(-1, G, (n,), device="cuda", dtype=torch.int32)
    g = P.group_rows(t, G)
    w = torch.randn(G, out, k, device="cuda").bfloat16()
    xs = [torch.randn(n, k, device="cuda").bfloat16() for _ in range(2)]
    ds = [torch.randn(n, out, device="cuda").bfloat16() for _ in range(2)]
    want = [(P.linear_typed(x, w, g),) + P.linear_typed_backward(d, x, w, g, bias=True) for x, d in zip(xs, ds)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for s, x, d in zip(streams, xs, ds):
            got.append((P.linear_typed(x, w, g, stream=s),) + P.linear_typed_backward(d, x, w, g, bias=True, stream=s))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_gradients_of_gradients_are_refused(torch):
    announce("gradients of gradients")
    g = P.group_rows(torch.zeros(8, dtype=torch.int32, device="cuda"), 1)
    x, w = torch.randn(8, 4, device="cuda", requires_grad=True), torch.randn(1, 4, 4, device="cuda", requires_grad=True)
    for y in (P.linear_typed(x, w, g), P.layer_norm(x)):
        d = torch.autograd.grad(y.square().sum(), x, create_graph=True)[0]
        with pytest.raises(RuntimeError):
            torch.autograd.grad(d.sum(), x)


def test_inputs_changed_since_are_refused_by_backward(torch):
    announce("inputs changed since")
    g = P.group_rows(torch.zeros(8, dtype=torch.int32, device="cuda"), 1)
    x, w = torch.randn(8, 4, device="cuda"), torch.randn(1, 4, 4, device="cuda", requires_grad=True)
    y = P.linear_typed(x, w, g)
    x.zero_()
    with pytest.raises(RuntimeError, match="modified"):
        torch.autograd.grad(y.sum(), w)
    y = P.linear_typed(x, w, g)
    g.order.copy_(g.order.flip(0))
    with pytest.raises(RuntimeError, match="modified"):
        torch.autograd.grad(y.sum(), w)


def test_group_rows_of_a_copy(torch):
    """Copies and pickles of groups have their own tensors."""
    import copy
    import pickle
    announce("copies of groups")
    g = P.group_rows(torch.randint(0, 3, (50,), device="cuda", dtype=torch.int32), 3)
    x, w = torch.randn(50, 8, device="cuda"), torch.randn(3, 5, 8, device="cuda")
    for c in (copy.deepcopy(g), pickle.loads(pickle.dumps(g))):
        assert c.order.data_ptr() != g.order.data_ptr() and c.c_view(50, 0).order == c.order.data_ptr()
        assert torch.equal(P.linear_typed(x, w, c), P.linear_typed(x, w, g))
