"""What the 8-bit operators' Python entry points refuse on a device."""
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu


def test_steps_that_require_a_gradient_are_refused():
    """A cache's steps are float32 and could: what is read with them has no gradient."""
    torch = require_gpu()
    announce("steps that require a gradient")
    c = P.HistoryCache.empty(8, 2, 16, 4)
    table = torch.arange(6, dtype=torch.int32).cuda().view(3, 2)
    q = torch.randn(3, 2, 16).cuda()
    c.scales.requires_grad_()
    for f in (lambda: P.cache_write(c, q, q, table), lambda: P.cache_read(c, table), lambda: P.cache_attend(c, q, table)):
        with pytest.raises(ValueError, match="gradient"):
            f()
    with torch.no_grad():
        P.cache_write(c, q, q, table)
        k, v = P.cache_read(c, table[:, :1], n=3)
    assert torch.equal(k, v) and ((k - q).abs() <= q.abs().amax(-1, keepdim=True) / 253).all()


def test_outputs_that_overlap_are_refused():
    """An output whose rows share memory cannot hold them."""
    torch = require_gpu()
    announce("outputs that overlap")
    c = P.HistoryCache.empty(8, 2, 16, 4)
    table = torch.arange(6, dtype=torch.int32).cuda().view(3, 2)
    q = torch.randn(3, 2, 16).cuda()
    room = torch.empty(24, 2, 16).cuda()
    one = torch.empty(1, 2, 16).cuda()
    for f in (lambda: P.cache_read(c, table, k=one.expand(24, 2, 16), v=room), lambda: P.cache_read(c, table, k=room, v=room[:, :1].expand(24, 2, 16)),
              lambda: P.cache_attend(c, q, table, out=one.expand(3, 2, 16)),
              lambda: P.cache_attend(c, q[:, None].contiguous(), table, out=one.expand(3, 1, 2, 16))):
        with pytest.raises(ValueError, match="overlap"):
            f()
    P.cache_attend(c, q[:1], table[:1], out=one.expand(1, 2, 16))
    P.cache_read(c, table[:1, :1], n=1, k=one, v=one.clone())
