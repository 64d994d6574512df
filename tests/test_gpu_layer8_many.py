"""Calls of more workgroups than one launch may have (2^32 threads)."""
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("places,group,bounded", [(1, 1, False), (1, 3, True), (300, 1, True), (2, 20, False)])
def test_attend_many_sequences(places, group, bounded):
    """2^24 sequences and a few: the kernels for few tokens, of one and of four wavefronts, of two row tiles."""
    torch = require_gpu()
    B, pages = (1 << 24) + 5, 1000
    announce("attend %d sequences of %d places, group %d" % (B, places, group))
    g = torch.Generator(device="cuda").manual_seed(places + group)
    c = P.HistoryCache.empty(pages, 1, 1, 1)
    c.data[..., 0] = torch.randint(-127, 128, (pages, 1, 2, 1), device="cuda", generator=g, dtype=torch.int8)
    c.scales[:] = 1.0
    first = torch.randint(0, pages, (B, min(places, 2)), device="cuda", generator=g, dtype=torch.int32)
    first[::17, 0] = -1
    table = first if places < 300 else torch.arange(300, dtype=torch.int32, device="cuda").expand(B, 300)
    q = torch.zeros(B, group, 1, device="cuda", dtype=torch.bfloat16)
    values = c.data[:, 0, 1, 0, 0].float()
    kw, see = {}, first
    if bounded and places == 300:           # one place each, anywhere in the table
        at = torch.randint(0, 300, (B,), device="cuda", generator=g)
        kw, see = dict(begin=at, end=at + 1), at[:, None]
    out, lse = P.cache_attend(c, q, table, return_lse=True, **kw)
    # all scores are 0: the mean of what is seen, within the rounding to bfloat16
    there = see >= 0
    count = there.sum(1)
    want = (values[see.long().clamp(min=0)] * there).sum(1) / count.clamp(min=1)
    assert ((out[..., 0].float() - want[:, None]).abs() <= 2.0 ** -8 * want.abs()[:, None] + 1e-30).all()
    assert ((lse.exp() - count[:, None]).abs() <= 1e-5).all()


def test_linear_i8_of_many_rows():
    """2^30 rows and a few, all of them the same bytes with a scale each."""
    torch = require_gpu()
    m, k = (1 << 30) + 37, 16
    announce("linear_i8 of %d rows" % m)
    x = torch.arange(-7, 9, dtype=torch.int8, device="cuda")
    w = torch.arange(100, 116, dtype=torch.int8, device="cuda")
    total = float((x.long() * w.long()).sum())
    scale = torch.rand(m, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    y = P.linear_i8(x.expand(m, k), scale, w[None], torch.ones(1, device="cuda"))
    assert torch.equal(y[:, 0], (scale * total).bfloat16())
