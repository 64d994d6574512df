"""Memory that is given for results counts as changed in place: a backward pass that kept it as an input raises."""
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu
N, D = 48, 64


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


def _calls(torch):
    """name -> call that writes to its argument, float32 [N, D]."""
    x, w = torch.randn(N, D, device="cuda"), torch.randn(2, D, D, device="cuda")
    g = P.group_rows(torch.randint(0, 2, (N,), device="cuda", dtype=torch.int32), 2)
    q, s = P.quant_rows(x)[:2]
    wq, ws = P.quant_rows(w[0])[:2]
    cache = P.HistoryCache.empty(4, 1, D, 16)
    table = torch.arange(4, device="cuda", dtype=torch.int32).view(4, 1)
    keys = torch.randn(16, 1, D, device="cuda")
    P.cache_write(cache, keys, keys, table)
    ids = torch.arange(N, device="cuda", dtype=torch.int32)
    omega = torch.ones(D, device="cuda")
    return {
        "linear_typed": lambda out: P.linear_typed(x, w, g, out=out),
        "norm_quant": lambda out: P.norm_quant(x, residual=x, out=out),
        "linear_i8": lambda out: P.linear_i8(q, s, wq, ws, out=out),
        "cache_attend": lambda out: P.cache_attend(cache, x.view(4, N // 4, D), table, out=out.view(4, N // 4, D)),
        "gather": lambda out: P.gather(ids, None, [(x, "node")], outs=[out]),
        "time_encode": lambda out: P.time_encode(x[:, 0].contiguous(), omega, omega, out=out),
    }


@pytest.mark.parametrize("name", ["linear_typed", "norm_quant", "linear_i8", "cache_attend", "gather", "time_encode"])
def test_outputs_count_as_changed(torch, name):
    announce("outputs count as changed: %s" % name)
    call = _calls(torch)[name]
    w = torch.randn(1, D, D, device="cuda", requires_grad=True)
    one = P.RowGroups(torch.tensor([0, N], device="cuda"))
    wide = torch.zeros(2 * N, D, device="cuda")
    for kept, out in ((wide[:N].clone(), None), (wide, wide[N:])):
        kept = kept[:N] if out is None else kept
        groups = one if out is None else P.RowGroups(torch.tensor([0, 2 * N], device="cuda"))
        y = P.linear_typed(kept, w, groups)
        with torch.no_grad():
            call(kept if out is None else out)
        assert bool(kept.any())
        with pytest.raises(RuntimeError, match="modified"):
            torch.autograd.grad(y.sum(), w)
    # and nothing else does
    y = P.linear_typed(wide, w, groups)
    call(torch.empty(N, D, device="cuda"))
    torch.autograd.grad(y.sum(), w)
