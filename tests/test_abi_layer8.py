"""The C ABI and the binding of the 8-bit operators: what they refuse before
they touch the device (every call here fails a host check, or has nothing to
do)."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2203_14883_amd as P
from paper_2203_14883_amd import binding as B

FAKE = 0x10000  # never dereferenced


def _norm(**kw):
    a = dict(x=FAKE, xs=64, r=None, rs=0, w=None, n=3, dim=64, dt=0, norm=1, eps=1e-6, q=FAKE, qs=64, scale=FAKE, sum=None, ss=0)
    a.update(kw)
    return P.lib().tgl_norm_quant(a["x"], a["xs"], a["r"], a["rs"], a["w"], a["n"], a["dim"], a["dt"], a["norm"], a["eps"],
                                  a["q"], a["qs"], a["scale"], a["sum"], a["ss"], None)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(dim=0), dict(dim=(1 << 20) + 1), dict(dt=2), dict(norm=2), dict(eps=-1.0), dict(eps=math.nan),
    dict(x=None), dict(q=None), dict(scale=None), dict(x=FAKE + 2), dict(x=FAKE + 1, dt=1), dict(r=FAKE + 1), dict(w=FAKE + 2),
    dict(q=FAKE + 8), dict(qs=72), dict(qs=48), dict(scale=FAKE + 1), dict(sum=FAKE, ss=63), dict(sum=FAKE + 2, ss=64),
])
def test_norm_quant_refuses(kw):
    assert _norm(**kw) == B.EINVAL


def test_norm_quant_of_nothing():
    assert _norm(n=0, x=None, q=None, scale=None) == 0


def _linear(**kw):
    a = dict(x=FAKE, xst=64, xs=FAKE, m=4, w=FAKE, wst=64, ws=FAKE, bias=None, n=8, k=64, out=FAKE, ost=8, dt=0)
    a.update(kw)
    return P.lib().tgl_linear_i8(a["x"], a["xst"], a["xs"], a["m"], a["w"], a["wst"], a["ws"], a["bias"], a["n"], a["k"],
                                 a["out"], a["ost"], a["dt"], None)


@pytest.mark.parametrize("kw", [
    dict(m=-1), dict(n=0), dict(n=(1 << 20) + 1), dict(k=0), dict(k=131073), dict(dt=-1), dict(x=None), dict(xs=None), dict(w=None),
    dict(ws=None), dict(out=None), dict(x=FAKE + 4), dict(w=FAKE + 8), dict(xst=72), dict(wst=8), dict(xst=-64), dict(xst=1 << 22),
    dict(wst=1 << 22), dict(xs=FAKE + 2), dict(bias=FAKE + 1), dict(out=FAKE + 2), dict(ost=7),
])
def test_linear_i8_refuses(kw):
    assert _linear(**kw) == B.EINVAL


def test_linear_i8_of_nothing():
    assert _linear(m=0, x=None, xs=None, out=None) == 0


def _cache(**kw):
    a = dict(data=FAKE, scales=FAKE, pages=8, page=4, heads=2, dim=50, reserved=0)
    a.update(kw)
    return B.c_cache(a["data"], a["scales"], a["pages"], a["page"], a["heads"], a["dim"], a["reserved"])


def _seqs(**kw):
    a = dict(table=FAKE, stride=5, seqs=3, pages=5, reserved=0, start=None, offsets=None)
    a.update(kw)
    return B.c_seqs(a["table"], a["stride"], a["seqs"], a["pages"], a["reserved"], a["start"], a["offsets"])


BAD_CACHE = [dict(data=None), dict(scales=None), dict(data=FAKE + 8), dict(scales=FAKE + 4), dict(pages=-1), dict(pages=2**31),
             dict(page=0), dict(page=3), dict(page=256), dict(heads=0), dict(heads=1025), dict(dim=0), dict(dim=257), dict(reserved=1)]
BAD_SEQS = [dict(table=None), dict(table=FAKE + 2), dict(stride=-1), dict(seqs=-1), dict(seqs=2**31), dict(pages=-1), dict(reserved=1),
            dict(start=FAKE + 4), dict(offsets=FAKE + 4)]


def _io(name, cache, seqs, **kw):
    a = dict(k=FAKE, v=FAKE, t=100, h=50, dt=0, n=6)
    a.update(kw)
    k, v = B.c_heads(a["k"], a["t"], a["h"]), B.c_heads(a["v"], a["t"], a["h"])
    return getattr(P.lib(), name)(C.byref(cache) if cache else None, C.byref(k), C.byref(v), a["dt"], a["n"],
                                  C.byref(seqs) if seqs else None, None)


@pytest.mark.parametrize("name", ["tgl_cache_write", "tgl_cache_read"])
def test_cache_io_refuses(name):
    for kw in BAD_CACHE:
        assert _io(name, _cache(**kw), _seqs()) == B.EINVAL, kw
    for kw in BAD_SEQS:
        assert _io(name, _cache(), _seqs(**kw)) == B.EINVAL, kw
    for kw in [dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(dt=2), dict(n=-1), dict(n=7), dict(v=FAKE + 1, dt=1)]:
        assert _io(name, _cache(), _seqs(), **kw) == B.EINVAL, kw
    assert _io(name, None, _seqs()) == B.EINVAL and _io(name, _cache(), None) == B.EINVAL
    assert _io(name, _cache(), _seqs(seqs=0), n=1) == B.EINVAL
    assert _io(name, _cache(), _seqs(), n=0, k=None, v=None) == 0
    assert _io(name, _cache(), _seqs(seqs=0, table=None), n=0) == 0
    if name == "tgl_cache_write":
        assert _io(name, _cache(), _seqs(), t=1 << 31) == B.EINVAL


def _attend(cache=None, seqs=None, **kw):
    a = dict(q=FAKE, out=FAKE, t=100, h=50, dt=0, heads=4, queries=1, end=None, scale=0.1, lse=None, ws=FAKE, bytes=1 << 40)
    a.update(kw)
    q, o = B.c_heads(a["q"], a["t"], a["h"]), B.c_heads(a["out"], a["t"], a["h"])
    c, s = cache or _cache(), seqs or _seqs()
    return P.lib().tgl_cache_attend(C.byref(c), C.byref(q), a["heads"], a["queries"], a["dt"], C.byref(s), a["end"], a["scale"],
                                    C.byref(o), a["lse"], a["ws"], a["bytes"], None)


def test_attend_refuses():
    for kw in BAD_CACHE:
        assert _attend(cache=_cache(**kw)) == B.EINVAL, kw
    for kw in BAD_SEQS + [dict(offsets=FAKE)]:
        assert _attend(seqs=_seqs(**kw)) == B.EINVAL, kw
    for kw in [dict(q=None), dict(out=None), dict(q=FAKE + 2), dict(out=FAKE + 1, dt=1), dict(dt=5), dict(heads=0), dict(heads=3),
               dict(heads=1026), dict(queries=0), dict(queries=2**31), dict(end=FAKE + 4), dict(lse=FAKE + 2), dict(scale=math.nan)]:
        assert _attend(**kw) == B.EINVAL, kw
    assert _attend(seqs=_seqs(seqs=2**30), queries=2) == B.EINVAL          # 2^33 rows of heads
    assert _attend(seqs=_seqs(seqs=0, table=None)) == 0


def _workspace(cache, seqs, heads=4, queries=1):
    return P.lib().tgl_cache_attend_workspace(C.byref(cache), C.byref(seqs), heads, queries)


def test_attend_workspace():
    assert _workspace(_cache(), _seqs()) == 0                              # 20 tokens: one chunk
    long = _seqs(seqs=1, pages=100_000, stride=100_000)
    need = _workspace(_cache(pages=100_000), long)
    assert need > 0
    assert _attend(cache=_cache(pages=100_000), seqs=long, bytes=need - 1) == B.ENOSPACE
    assert _attend(cache=_cache(pages=100_000), seqs=long, ws=None) == B.ENOSPACE
    assert _attend(cache=_cache(pages=100_000), seqs=long, ws=FAKE + 4) == B.EINVAL
    assert _workspace(_cache(), _seqs(), heads=3) == 0 and _workspace(_cache(dim=0), long) == 0
    # positions beyond 32 bits
    assert _workspace(_cache(page=128), _seqs(seqs=1, pages=2**31 - 1, stride=2**31)) > 0


def test_python_refuses_host_tensors_and_gradients():
    torch = pytest.importorskip("torch")
    x = torch.randn(4, 32)
    c = P.HistoryCache.empty(8, 2, 16, 4, device="cpu")
    assert c.num_pages == 8 and c.heads == 2 and c.page_tokens == 4 and c.data.shape == (8, 2, 2, 4, 16)
    q = torch.zeros(3, 2, 16)
    t = torch.zeros(3, 2, dtype=torch.int32)
    for f in (lambda: P.norm_quant(x), lambda: P.quant_rows(x), lambda: P.linear_i8(x.to(torch.int8), x[:, 0], x.to(torch.int8), x[:, 0]),
              lambda: P.cache_write(c, q, q, t), lambda: P.cache_read(c, t), lambda: P.cache_attend(c, q, t)):
        with pytest.raises((ValueError, RuntimeError)):
            f()
    for bad in (dict(page_tokens=3), dict(page_tokens=256), dict(dim=0), dict(dim=257), dict(heads=0)):
        with pytest.raises(ValueError):
            P.HistoryCache.empty(**{**dict(num_pages=4, heads=2, dim=16, page_tokens=4, device="cpu"), **bad})
    with pytest.raises(ValueError):
        P.HistoryCache(c.data[:, :, :, :, :8], c.scales, 8)
    with pytest.raises(Exception):
        c.dim = 3                       # a cache does not change under its view


def test_oracle_of_a_hand_written_page():
    """Steps and bytes worked out by hand."""
    from oracle import layer8 as O
    c = O.Cache(np.zeros((2, 1, 2, 4, 16), np.int8), np.zeros((2, 1, 2), np.float32), 3)
    table = np.array([[1]], np.int32)
    k = np.array([[[127.0, -63.6, 0.4]], [[1.0, 2.0, -3.5]]], np.float32)
    c.write(k, np.zeros_like(k), table, [0], [0, 2])
    assert c.scales[1, 0, 0] == 1 and c.scales[1, 0, 1] == 0 and c.scales[0, 0, 0] == 0
    assert c.data[1, 0, 0, :2, :3].tolist() == [[127, -64, 0], [1, 2, -4]]          # -3.5 rounds to even
    c.write(np.array([[[254.0, 5.0, 3.0]]], np.float32), np.zeros((1, 1, 3), np.float32), table, [2], [0, 1])
    assert c.scales[1, 0, 0] == 2
    assert c.data[1, 0, 0, :3, :3].tolist() == [[64, -32, 0], [0, 1, -2], [127, 2, 2]]    # 63.5, 0.5, 2.5 and 1.5 to even
    out, lse = c.attend(np.zeros((1, 1, 1, 3)), table, None, [3], 1.0)
    assert np.allclose(out, 0) and np.allclose(lse, math.log(3))
    k2, _, ok = c.tokens(table, 0, [0, 4])
    assert ok.tolist() == [True, False] and k2[0, 0].tolist() == [128.0, -64.0, 0.0]


def test_oracle_norm_is_a_norm():
    from oracle import layer8 as O
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((5, 300)).astype(np.float32), rng.standard_normal(300).astype(np.float32)
    q, s, h = O.norm_quant(x, x, w, 0.0)
    want = h * w / np.sqrt((h.astype(np.float64) ** 2).mean(1, keepdims=True))
    assert np.abs(q * s[:, None] - want).max() <= 0.5001 * s.max()
    assert np.abs(q).max(1).tolist() == [127] * 5
