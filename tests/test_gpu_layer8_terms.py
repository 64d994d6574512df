"""Attention over an 8-bit cache where a row's terms differ by many orders of
magnitude, against float64 and within bounds made of the row's own terms."""
import math

import numpy as np
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu
from oracle import layer8 as O
from test_gpu_layer8 import HALF, TYPES, _cache, _host, _tables, _torch_type, _up

pytestmark = pytest.mark.gpu


def _bounds(dtype, oc, qh, table, begin, end, scale, want):
    """Bound of every output's error from the terms p_j |v_j| that it sums.

    With e a bound of the error of a score: a query element is held to 2^-24 of
    the row's largest; products, sums of at most 256 of them (16 in turn and a
    tree) and the exponential's argument are float32, 24 roundings at the most.
    A mean of values whose weights are each off by a factor exp(+-2 e) moves by 2 e
    of sum p |v|.  Weights are held to 2^-22 of themselves, and to 2^-36 of the row's
    largest p times step; exponentials to 2^-21; sums are float32, length / 16
    terms in turn at the least parallel."""
    B, T, H, D = qh.shape
    g = H // oc.data.shape[1]
    all_ = table.shape[1] * oc.P
    tol = np.zeros(qh.shape)
    for b in range(B):
        a = 0 if begin is None else max(0, int(begin[b]))
        e = all_ if end is None else min(all_, int(end[b]))
        k, v, ok = oc.tokens(table, b, range(a, max(a, e)))
        pages = [oc.page(table, b, p // oc.P) for p in range(a, max(a, e))]
        for t in range(T):
            see = ok.copy()
            see[max(0, (all_ if end is None else int(end[b])) - (T - 1 - t) - a):] = False
            if not see.any():
                continue
            step = oc.scales[np.array(pages)[see]][:, :, 1].astype(np.float64)
            for h in range(H):
                ks, vs, q = k[see, h // g], v[see, h // g], qh[b, t, h].astype(np.float64)
                s = ks @ q * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                err = abs(scale) * HALF * (np.abs(q).max() * np.abs(ks).sum(1).max() + 24 * (np.abs(ks) @ np.abs(q)).max())
                sums = p @ np.abs(vs)
                tol[b, t, h] = sums * (2 * err + 2.0 ** -20 + (16 + len(p) / 16) * HALF) + len(p) * 127 * 2.0 ** -36 * (p * step[:, h // g]).max()
    return tol + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)


def _check(torch, dtype, c, oc, q, qh, table, begin, end, scale):
    kw = {}
    if begin is not None:
        kw["begin"] = torch.from_numpy(np.asarray(begin, np.int64)).cuda()
    if end is not None:
        kw["end"] = torch.from_numpy(np.asarray(end, np.int64)).cuda()
    out = _host(P.cache_attend(c, q, torch.from_numpy(table).cuda(), scale=scale, **kw))
    with np.errstate(over="ignore"):
        want, _ = oc.attend(qh, table, begin, end, scale)
    tol = _bounds(dtype, oc, qh, table, begin, end, scale, want)
    assert np.isfinite(out).all()
    over = np.abs(out - want) / np.maximum(tol, 1e-300)
    assert np.all(np.abs(out - want) <= tol), "largest error %.3g of its bound" % over.max()
    return out


# what a call of so many places, rows and sequences runs: few tokens; one wavefront; four; chunks; two row tiles
LAYOUTS = [(1, 1, 1, 10, 3), (4, 1, 1, 48, 2), (1, 1, 3, 60, 2), (16, 2, 3, 64, 2), (1, 1, 2, 300, 2), (4, 1, 2, 300, 3), (16, 2, 2, 300, 2),
           (64, 1, 1, 300, 1), (16, 1, 2, 3000, 1), (2, 1, 1, 2000, 1), (16, 1, 20, 200, 2), (4, 1, 40, 1500, 1)]


@pytest.mark.parametrize("page,heads,group,length,B", LAYOUTS)
def test_attend_bfloat16_small_elements_beside_a_large_one(page, heads, group, length, B):
    """One column of the query is 4096 times the others, where every key is 0: the others make the scores."""
    torch = require_gpu()
    announce("bfloat16 query with an outlier, page %d rows %d tokens %d" % (page, group, length))
    rng = np.random.default_rng(length + group)
    D, need = 64, -(-length // page)
    c, oc = _cache(rng, torch, B * need, heads, page, D)
    oc.data[:, :, 0, :, 5] = 0
    c.data[:, :, 0, :, 5] = 0
    table = _tables(rng, np.full(B, need), need, B * need)
    qh = rng.standard_normal((B, 1, heads * group, D))
    qh[..., 5] = 4096
    q, qh = _up(torch, qh, "bf16")
    _check(torch, "bf16", c, oc, q, qh, table, None, np.full(B, length), 1 / math.sqrt(D))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,group,length", [(1, 1, 12), (1, 3, 60), (16, 3, 64), (16, 2, 200), (4, 2, 200), (1, 2, 200), (16, 20, 200)])
def test_attend_weights_whose_terms_cancel(page, group, length, dtype):
    """A last token that takes away what the others add up to: what is left shows how the weights are held."""
    torch = require_gpu()
    announce("terms that cancel, page %d rows %d tokens %d %s" % (page, group, length, dtype))
    rng = np.random.default_rng(length * 3 + group)
    D, need = 32, -(-length // page)
    c, oc = _cache(rng, torch, need, 1, page, D)
    oc.scales[..., 0] = 2.0 ** -12
    oc.scales[..., 1] = 0.5
    oc.data[:, 0, 0] = rng.integers(-3, 4, oc.data[:, 0, 0].shape)
    table = _tables(rng, np.array([need]), need, need)
    qh = np.ones((1, 1, group, D)) * (1 + np.arange(group)[:, None] % 2)
    last, row = oc.page(table, 0, (length - 1) // page), (length - 1) % page
    oc.data[last, 0, 0, row] = 127
    scale = 0.75 * math.log(length) / (127 * D * 2.0 ** -12)         # its weight is length^0.75 of the others'
    q, qh = _up(torch, qh, dtype)
    k, v, _ = oc.tokens(table, 0, range(length))
    p = np.exp((k[:, 0] @ qh[0, 0, 0].astype(np.float64)) * scale)
    take = -(p[:-1] @ v[:-1, 0]) / p[-1] / 0.5                      # so the terms of every other row cancel
    oc.data[last, 0, 1, row, :D] = np.clip(np.rint(take), -127, 127)
    c.data.copy_(torch.from_numpy(oc.data))
    c.scales.copy_(torch.from_numpy(oc.scales))
    _check(torch, dtype, c, oc, q, qh, table, None, np.array([length]), scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ratio", [2.0 ** 12, 2.0 ** 24, 2.0 ** 32, 2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("page,heads,group,length,B", LAYOUTS)
def test_attend_a_large_step_without_weight(page, heads, group, length, B, ratio, dtype):
    """A first page whose step is ratio times the others' and whose scores lie so far below that its terms are as small as theirs."""
    torch = require_gpu()
    announce("large step %g, page %d rows %d tokens %d %s" % (ratio, page, group, length, dtype))
    rng = np.random.default_rng(length + group)
    D, need = 32, -(-length // page)
    c, oc = _cache(rng, torch, B * need, heads, page, D)
    oc.scales[:] = 2.0 ** -6
    oc.data[:, :, 0] = rng.integers(-9, 10, oc.data[:, :, 0].shape)
    oc.data[:, :, 1, :, :D] = 100
    table = _tables(rng, np.full(B, need), need, B * need)
    qh = np.ones((B, 1, heads * group, D))
    scale = 1 / math.sqrt(D)
    below = (math.log(ratio) + 3) / (D * scale)
    for b in range(B):
        for at in (0, need // 2):           # the first page, and one that comes later
            oc.data[table[b, at], :, 0] = -127
            oc.scales[table[b, at], :, 0] = below / 127
            oc.scales[table[b, at], :, 1] *= ratio
    c.data.copy_(torch.from_numpy(oc.data))
    c.scales.copy_(torch.from_numpy(oc.scales))
    q, qh = _up(torch, qh, dtype)
    _check(torch, dtype, c, oc, q, qh, table, None, np.full(B, length), scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,group,length,B", LAYOUTS)
def test_attend_terms_of_any_size(page, heads, group, length, B, dtype):
    """Steps from 1e-20 to 1e20 in no order, scores up to 40 either way: any token may make the output."""
    torch = require_gpu()
    announce("terms of any size, page %d rows %d tokens %d %s" % (page, group, length, dtype))
    rng = np.random.default_rng(7 * length + group)
    D, need = 16, -(-length // page)
    c, oc = _cache(rng, torch, B * need, heads, page, D)
    oc.scales[..., 1] = 10.0 ** rng.uniform(-20, 20, oc.scales[..., 1].shape)
    oc.scales[..., 0] = 40.0 / 127 / D
    oc.data[:, :, 0, :, :D] = rng.integers(-127, 128, oc.data.shape[:2] + (page, 1))
    c.data.copy_(torch.from_numpy(oc.data))
    c.scales.copy_(torch.from_numpy(oc.scales))
    table = _tables(rng, np.full(B, need), need, B * need)
    q, qh = _up(torch, rng.uniform(0.2, 1, (B, 1, heads * group, 1)) * np.ones(D), dtype)
    _check(torch, dtype, c, oc, q, qh, table, None, np.full(B, length), 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("up", [1, -1])
@pytest.mark.parametrize("page,group,length", [(1, 2, 60), (16, 2, 300), (4, 1, 900), (2, 2, 3000), (16, 9, 300)])
def test_attend_scores_that_rise_while_steps_fall(page, group, length, up, dtype):
    """Scores grow along the history by 75 in all while steps shrink as fast, or the other way."""
    torch = require_gpu()
    announce("rising scores %d, page %d rows %d tokens %d %s" % (up, page, group, length, dtype))
    rng = np.random.default_rng(length)
    D, need = 16, -(-length // page)
    c, oc = _cache(rng, torch, need, 1, page, D)
    along = np.linspace(0, 1, need) if up > 0 else np.linspace(1, 0, need)
    table = np.arange(need, dtype=np.int32)[None]
    oc.data[:, 0, 0, :, :D] = 127
    oc.scales[:, 0, 0] = np.maximum(along, 1e-3) * 75 / 127 / D
    oc.scales[:, 0, 1] = np.exp(-75 * along + 20)
    c.data.copy_(torch.from_numpy(oc.data))
    c.scales.copy_(torch.from_numpy(oc.scales))
    q, qh = _up(torch, np.ones((1, 1, group, D)), dtype)
    _check(torch, dtype, c, oc, q, qh, table, None, np.array([length]), 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,group,T,length", [(1, 1, 3, 50), (1, 1, 3, 300), (4, 2, 5, 300), (16, 1, 3, 146), (16, 4, 9, 290), (1, 1, 40, 200), (1, 2, 3, 3000)])
def test_attend_a_later_event_changes_no_earlier_query(page, group, T, length, dtype):
    """The newest tokens have steps 2^40 times the others': queries that do not see them are as they are without."""
    torch = require_gpu()
    announce("later event, page %d rows %d queries %d tokens %d %s" % (page, group, T, length, dtype))
    rng = np.random.default_rng(length + T)
    D, need = 48, -(-length // page)
    c, oc = _cache(rng, torch, need, 1, page, D)
    table = np.arange(need, dtype=np.int32)[None]
    oc.scales[:] = 1 / 64
    new = (length - 1) // page              # the page that the newest token is on
    oc.scales[new] = (1 / 64, 2.0 ** 34)
    c.scales.copy_(torch.from_numpy(oc.scales))
    q, qh = _up(torch, rng.standard_normal((1, T, group, D)), dtype)
    out = _check(torch, dtype, c, oc, q, qh, table, None, np.array([length]), 1 / math.sqrt(D))
    for t in range(T):
        if length - (T - 1 - t) <= new * page:                              # sees none of that page
            _check(torch, dtype, c, oc, q[:, t:t + 1], qh[:, t:t + 1], table, None, np.array([length - (T - 1 - t)]), 1 / math.sqrt(D))
            assert np.abs(out[0, t]).max() < 100


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,group,length,B", LAYOUTS)
def test_attend_values_near_the_largest_float(page, heads, group, length, B, dtype):
    """A mean of values near 1.7e38 is such a value, however many there are."""
    torch = require_gpu()
    announce("large values, page %d rows %d tokens %d %s" % (page, group, length, dtype))
    rng = np.random.default_rng(length + 2 * group)
    D, need = 32, -(-length // page)
    c, oc = _cache(rng, torch, B * need, heads, page, D)
    oc.scales[..., 1] = 2.0 ** 120
    oc.data[:, :, 1, :, :D] = rng.integers(90, 128, oc.data[:, :, 1, :, :D].shape)
    c.data.copy_(torch.from_numpy(oc.data))
    c.scales.copy_(torch.from_numpy(oc.scales))
    table = _tables(rng, np.full(B, need), need, B * need)
    q, qh = _up(torch, rng.standard_normal((B, 1, heads * group, D)), dtype)
    _check(torch, dtype, c, oc, q, qh, table, None, np.full(B, length), 1 / math.sqrt(D))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,group,T,length", [(1, 1, 1, 1), (1, 1, 1, 10), (4, 1, 1, 60), (1, 2, 1, 16), (1, 3, 1, 60), (16, 2, 2, 64), (1, 2, 1, 300),
                                                 (16, 2, 1, 300), (4, 1, 1, 3000), (16, 20, 1, 200)])
def test_attend_scores_that_are_no_numbers(page, group, T, length, dtype):
    """A row whose largest score is not finite is NaN, whichever sign made it; one that sees nothing is 0."""
    torch = require_gpu()
    announce("scores without end, page %d rows %d x %d tokens %d %s" % (page, group, T, length, dtype))
    D, need = 16, -(-length // page)
    B = 4
    near = 7 * (2.0 ** -20 + (16 + length / 16) * HALF)                     # bfloat16: rounded to 7 itself
    data = torch.zeros(need, 1, 2, page, D, dtype=torch.int8).cuda()
    data[:, 0, 0] = 3
    data[:, 0, 1] = 7
    c = P.HistoryCache(data, torch.ones(need, 1, 2).cuda(), D)
    table = torch.arange(need, dtype=torch.int32).cuda().expand(B, need)
    end = torch.tensor([length, 0, length, length + T - 1]).cuda()
    for value, finite in [(math.inf, 0), (-math.inf, 0), (math.nan, 0), (2.0 ** 127, 0), (-2.0 ** 127, 0), (1.0, 1)]:
        for scale in (1.0, -1.0):
            q = torch.ones(B, T, group, D).cuda().to(_torch_type(torch, dtype))
            q[:2, :, 0] = value
            q[3, -1, group - 1, 11] = value
            out, lse = P.cache_attend(c, q, table, end=end, scale=scale, return_lse=True)
            out, lse = _host(out), lse.cpu().numpy()
            what = "%g, scale %g" % (value, scale)
            assert (out[1] == 0).all() and np.isneginf(lse[1]).all(), what
            if finite:
                assert (np.abs(out[[0, 2], -1] - 7) <= near).all(), what
                continue
            assert np.isnan(out[0, -1, 0]).all() and np.isnan(lse[0, -1, 0]), what
            assert (np.abs(out[2, -1] - 7) <= near).all() and np.isfinite(lse[2, -1]).all(), what
            if not np.isfinite(value):
                assert np.isnan(out[3, -1, group - 1]).all() and np.isnan(lse[3, -1, group - 1]), what


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,group,length", [(1, 1, 10), (1, 3, 60), (1, 2, 300), (4, 2, 300), (1, 1, 3000)])
def test_attend_a_score_far_below_has_no_weight(page, group, length, dtype):
    """Scores of minus infinity beside finite ones weigh nothing; a hidden infinite one does not count."""
    torch = require_gpu()
    announce("scores far below, page %d rows %d tokens %d %s" % (page, group, length, dtype))
    D, need = 16, -(-length // page)
    data = torch.zeros(need, 1, 2, page, D, dtype=torch.int8).cuda()
    data[:, 0, 0] = 100
    data[:, 0, 1] = 7
    near = 7 * (2.0 ** -20 + (16 + length / 16) * HALF)
    scales = torch.full((need, 1, 2), 1e-36).cuda()
    scales[..., 1] = 1.0
    scales[::2, 0, 0] = 1e5
    scales[::2, 0, 1] = 1000.0
    c = P.HistoryCache(data, scales, D)
    table = torch.arange(need, dtype=torch.int32).cuda()[None]
    q = torch.full((1, group, D), -1e37).cuda().to(_torch_type(torch, dtype))
    out, lse = P.cache_attend(c, q, table, scale=1.0, return_lse=True)
    assert ((out.float() - 7).abs() <= near).all() and torch.isfinite(lse).all()
    table[0, ::2] = -1
    out = P.cache_attend(c, -q, table, scale=1.0)
    assert ((out.float() - 7).abs() <= near).all()
