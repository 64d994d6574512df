"""Kernels and branches that only larger calls of the 8-bit operators reach.
Every case names the kernel that it is there for, and fails if another runs."""
import warnings

import numpy as np
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu
from oracle import layer8 as O
from test_gpu_layer8 import HALF, TYPES, _attend, _cache, _host, _tables, _torch_type, _up

pytestmark = pytest.mark.gpu
NAME = {"f32": "float", "bf16": "tgl::bf16_t"}


def _ran(torch, call):
    """What a call returns, and the library's kernels that it ran."""
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with profile(activities=[ProfilerActivity.CUDA]) as p:
            out = call()
            torch.cuda.synchronize()
    names = {e.key.split("(anonymous namespace)::")[1].split("(")[0] for e in p.key_averages() if "tgl::" in e.key}
    return out, names


# ---- product ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k,bias,kernel", [
    (2100, 2050, 395, True, "linear_tile_kernel<%s, 128, 128, 2, 2>"), (12_000, 1000, 777, False, "linear_tile_kernel<%s, 128, 128, 2, 2>"),
    (33_000, 120, 96, True, "linear_tile_kernel<%s, 128, 128, 2, 2>"), (1, 33_000, 48, True, "linear_tile_kernel<%s, 128, 128, 2, 2>"),
    (2176, 2048, 512, False, "linear_tile_kernel<%s, 128, 128, 2, 2>"), (2049, 2305, 1, True, "linear_tile_kernel<%s, 128, 128, 2, 2>"),
    (3585, 3500, 300, True, "linear_tile_kernel<%s, 256, 256, 8, 2>"), (1537, 1409, 200, True, "linear_tile_kernel<%s, 64, 64, 1, 4>"),
    (33, 4100, 640, False, "linear_tile_kernel<%s, 64, 64, 1, 4>"), (5, 900, 2000, True, "linear_small_kernel<%s, 8, 1>"),
    (1, 20_000, 600, False, "linear_small_kernel<%s, 4, 1>"), (7, 100, 64, True, "linear_small_kernel<%s, 1, 1>"),
    (40, 700, 2000, True, "linear_small_kernel<%s, 8, 2>"), (40, 700, 300, False, "linear_small_kernel<%s, 4, 2>"), (20, 64, 40, True, "linear_small_kernel<%s, 1, 2>"),
])
def test_product_kernels(m, n, k, bias, kernel, dtype):
    torch = require_gpu()
    announce("product %d x %d x %d %s" % (m, n, k, dtype))
    rng = np.random.default_rng(m + 3 * n + 5 * k)
    kp = O.round16(k)
    xb = rng.integers(-128, 128, (m, kp)).astype(np.int8)
    wb = rng.integers(-128, 128, (n, kp)).astype(np.int8)
    xs, ws = rng.uniform(0.5, 2, m).astype(np.float32), rng.uniform(0.01, 0.02, n).astype(np.float32)
    b = (100 * rng.standard_normal(n)).astype(np.float32) if bias else None
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    x, w, s, t, c = up(xb)[:, :k], up(wb)[:, :k], up(xs), up(ws), None if b is None else up(b)
    room = torch.full((m + 1, n + 3), 5.0).cuda().to(_torch_type(torch, dtype))
    y, names = _ran(torch, lambda: P.linear_i8(x, s, w, t, c, out=room[:m, 2:n + 2]))
    assert names == {kernel % NAME[dtype]}
    want = O.linear_i8(xb[:, :k], xs, wb[:, :k], ws, b)
    prod = want if b is None else want - b
    tol = 4 * HALF * (np.abs(prod) + (0 if b is None else np.abs(b))) + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    assert np.all(np.abs(_host(y) - want) <= tol + 1e-30)
    assert (room[m] == 5).all() and (room[:, :2] == 5).all() and (room[:, n + 2:] == 5).all()


# ---- rows -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,dim,kernel", [
    (16_500, 100, "norm_kernel<%s, 64, 1>"), (20_001, 600, "norm_kernel<%s, 64, 2>"), (4100, 1030, "norm_kernel<%s, 256, 1>"),
    (8300, 2100, "norm_kernel<%s, 256, 2>"), (4097, 4100, "norm_kernel<%s, 256, 4>"), (4099, 8200, "norm_long_kernel<%s>"),
])
def test_norm_of_more_rows_than_workgroups_take_at_once(n, dim, kernel, dtype):
    torch = require_gpu()
    announce("norm of %d rows of %d %s" % (n, dim, dtype))
    rng = np.random.default_rng(n)
    size = np.exp(rng.uniform(-3, 3, (n, 1))).astype(np.float32)
    x, xh = _up(torch, size * rng.standard_normal((n, dim), dtype=np.float32), dtype)
    r, rh = _up(torch, rng.standard_normal((n, dim), dtype=np.float32), dtype)
    w, wh = _up(torch, 1 + 0.2 * rng.standard_normal(dim))
    (q, scale, h), names = _ran(torch, lambda: P.norm_quant(x, w, residual=r, eps=1e-5))
    assert names == {kernel % NAME[dtype]}
    oq, oscale, oh = O.norm_quant(xh, rh, wh, 1e-5)
    assert np.array_equal(q.cpu().numpy(), oq)
    np.testing.assert_allclose(scale.cpu().numpy(), oscale, rtol=(dim / 64 + 24) * HALF)
    assert np.array_equal(_host(h), oh if dtype == "f32" else O.to_bf16(oh))


# ---- cache ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,dim,seqs,hi,kept,lanes,pairs", [
    (1, 2, 50, 70_000, 1, 0, 16, 4), (1, 3, 50, 70_000, 1, 0, 16, 2), (16, 4, 64, 1500, 300, 40, 64, 8), (32, 8, 100, 150, 900, 100, 256, 8),
    (64, 4, 256, 60, 2000, 300, 512, 4), (32, 8, 100, 40, 1600, 100, 256, 2), (32, 8, 100, 48, 2000, 100, 256, 4), (4, 1, 128, 9000, 40, 9, 64, 2),
])
def test_cache_write_of_many_tokens(page, heads, dim, seqs, hi, kept, lanes, pairs, dtype):
    """Several keys and values of a page one after another: the same bytes as calls of few sequences, which take one
    each, and for some of the sequences the oracle's."""
    torch = require_gpu()
    announce("write %d sequences, page %d heads %d dim %d %s" % (seqs, page, heads, dim, dtype))
    rng = np.random.default_rng(seqs + page)
    start = rng.integers(0, kept + 1, seqs)
    new = np.full(seqs, 1) if hi == 1 else rng.integers(0, hi + 1, seqs)
    need = -(-(start + new) // page)
    pages = int(need.sum()) + 3
    table = _tables(rng, need, int(need.max()), pages)
    # the rule that the library shares work by: wavefronts that fill the card four times
    n = int(new.sum())
    items, parts, want = ((n + seqs * (2 * page - 2)) // page) + 1, 2 * heads, 1
    while want < 8 and parts % 2 == 0 and items * (parts // 2) * lanes >= 1 << 20:
        parts, want = parts // 2, 2 * want
    assert want == pairs
    g = torch.Generator(device="cuda").manual_seed(seqs)
    data = torch.randint(-127, 128, (pages, heads, 2, page, O.round16(dim)), device="cuda", generator=g, dtype=torch.int8)
    data[..., dim:] = 0
    scales = torch.exp(torch.randn(pages, heads, 2, device="cuda", generator=g)) / 64
    kv = torch.randn(n, 2, heads, dim, device="cuda", generator=g) * torch.exp(torch.randn(n, 1, 1, 1, device="cuda", generator=g))
    kv = kv.to(_torch_type(torch, dtype))
    offsets = np.concatenate([[0], np.cumsum(new)])
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    tab, st, of = up(table), up(start), up(offsets)
    c, d = (P.HistoryCache(data.clone(), scales.clone(), dim) for _ in range(2))
    _, names = _ran(torch, lambda: P.cache_write(c, kv[:, 0], kv[:, 1], tab, start=st, offsets=of))
    assert names == {"write_kernel<%s, %d>" % (NAME[dtype], lanes)}
    step = max(1, (1 << 19) // max(1, lanes * heads * (items // seqs + 1)))
    for b in range(0, seqs, step):
        e = min(seqs, b + step)
        t0, t1 = int(offsets[b]), int(offsets[e])
        P.cache_write(d, kv[t0:t1, 0], kv[t0:t1, 1], tab[b:e], start=st[b:e].contiguous(), offsets=of[b:e + 1] - t0)
    assert torch.equal(c.data, d.data)
    assert torch.equal(c.scales, d.scales)
    for b in np.unique(np.concatenate([rng.integers(0, seqs, 5), [0, seqs - 1]])):
        own = table[b][table[b] >= 0]
        oc = O.Cache(data[own].cpu().numpy(), scales[own].cpu().numpy(), dim)
        t0, t1 = int(offsets[b]), int(offsets[b + 1])
        oc.write(_host(kv[t0:t1, 0]), _host(kv[t0:t1, 1]), np.arange(len(own), dtype=np.int32)[None], start[b:b + 1], np.array([0, t1 - t0]))
        np.testing.assert_array_equal(c.data[own].cpu().numpy(), oc.data)
        np.testing.assert_array_equal(c.scales[own].cpu().numpy(), oc.scales)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,dim,seqs,hi", [(16, 2, 50, 700, 120), (1, 1, 16, 9000, 130), (64, 4, 128, 40, 2000), (4, 3, 7, 20_000, 9), (128, 1, 30, 3, 90_000)])
def test_cache_read_of_many_tokens(page, heads, dim, seqs, hi, dtype):
    """Several tokens a workgroup, of sequences of all lengths, none among them."""
    torch = require_gpu()
    announce("read %d sequences, page %d heads %d dim %d %s" % (seqs, page, heads, dim, dtype))
    rng = np.random.default_rng(seqs + page)
    count = rng.integers(0, hi + 1, seqs) * (rng.random(seqs) < 0.7)
    start = rng.integers(0, 2 * page + 1, seqs)
    need = -(-(start + count) // page)
    pages, width = int(need.sum()) + 5, int(need.max()) + 1
    table = _tables(rng, need, width, pages)
    table[rng.random(table.shape) < 0.05] = -1
    c, oc = _cache(rng, torch, pages, heads, page, dim)
    offsets = np.concatenate([[0], np.cumsum(count)])
    n = int(offsets[-1])
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    k, v = P.cache_read(c, up(table), start=up(start), offsets=up(offsets), n=n, out_dtype=_torch_type(torch, dtype))
    seq = np.repeat(np.arange(seqs), count)
    pos = start[seq] + np.arange(n) - offsets[seq]

    def held(seq, pos):
        at = table[seq, pos // page]
        got = oc.data[at, :, :, pos % page, :dim].astype(np.float32) * oc.scales[at][..., None]
        got[at < 0] = 0
        return got if dtype == "f32" else O.to_bf16(got)

    want = held(seq, pos)
    np.testing.assert_array_equal(_host(k), want[:, :, 0])
    np.testing.assert_array_equal(_host(v), want[:, :, 1])
    # as many of each, without offsets
    per = min(width * page, max(1, 40_000 // seqs))
    k, v = P.cache_read(c, up(table), n=per * seqs, out_dtype=_torch_type(torch, dtype))
    want = held(np.repeat(np.arange(seqs), per), np.tile(np.arange(per), seqs))
    np.testing.assert_array_equal(_host(k), want[:, :, 0])
    np.testing.assert_array_equal(_host(v), want[:, :, 1])


# ---- attention --------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,group,dim,T,length,kernels", [
    (64, 1, 2, 200, 1, 20_000, ["attend_kernel<%s, 16, 2, 4, 1>", "attend_join_kernel<%s, 16, 64>"]),
    (16, 1, 3, 256, 1, 3000, ["attend_kernel<%s, 16, 2, 4, 1>", "attend_join_kernel<%s, 1, 64>"]),
    (8, 1, 2, 128, 1, 20_000, ["attend_kernel<%s, 8, 1, 4, 1>", "attend_join_kernel<%s, 16, 32>"]),
    (32, 2, 1, 100, 1, 2000, ["attend_kernel<%s, 8, 2, 4, 1>", "attend_join_kernel<%s, 1, 32>"]),
    (1, 1, 1, 50, 1, 9000, ["attend_kernel<%s, 4, 0, 4, 1>", "attend_join_kernel<%s, 16, 16>"]),
    (2, 1, 20, 20, 1, 5000, ["attend_kernel<%s, 2, 0, 4, 2>", "attend_join_kernel<%s, 1, 16>"]),
    (16, 1, 2, 128, 30, 40_000, ["attend_kernel<%s, 8, 2, 4, 2>", "attend_join_kernel<%s, 16, 32>"]),
    (1, 2, 3, 64, 1, 60, ["attend_kernel<%s, 4, 0, 1, 1>"]), (4, 2, 4, 32, 1, 64, ["attend_kernel<%s, 2, 1, 1, 1>"]),
    (16, 2, 4, 128, 1, 64, ["attend_kernel<%s, 8, 2, 1, 1>"]), (64, 2, 2, 200, 2, 64, ["attend_kernel<%s, 16, 2, 1, 1>"]),
    (1, 2, 1, 50, 1, 64, ["attend_few_kernel<%s, 4>"]), (2, 2, 2, 100, 1, 16, ["attend_few_kernel<%s, 8>"]), (8, 1, 1, 256, 2, 16, ["attend_few_kernel<%s, 16>"]),
])
def test_attend_kernels(page, heads, group, dim, T, length, kernels, dtype):
    torch = require_gpu()
    announce("attend page %d heads %d group %d dim %d queries %d length %d %s" % (page, heads, group, dim, T, length, dtype))
    rng = np.random.default_rng(length + dim)
    c, q, tab, kw, out = _attend(torch, rng, dtype, page, heads, group, dim, T, [length], holes=0.02, extra=0)
    again, names = _ran(torch, lambda: P.cache_attend(c, q, tab, **kw))
    assert names == {k % NAME[dtype] for k in kernels}
    assert torch.equal(again, out)
