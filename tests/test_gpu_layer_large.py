"""Rows and weights of more than 2^31 elements, and layer norm's gradients for every set of leaves."""
import itertools

import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


def _whole(torch, *shape, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, device="cuda", generator=g).bfloat16()


def test_rows_beyond_32_bits(torch):
    """600,000 rows of 4096: a block of 1000 whole-numbered rows again and again, whose results are exact."""
    announce("typed products of 600,000 x 4096")
    times, block, k, out = 600, 1000, 4096, 64
    x, d, w = _whole(torch, block, k, seed=1), _whole(torch, block, out, seed=2), _whole(torch, 2, out, k, seed=3)
    t = torch.randint(-1, 2, (block,), device="cuda", generator=torch.Generator("cuda").manual_seed(4), dtype=torch.int32)
    big, big_d = x.repeat(times, 1), d.repeat(times, 1)
    assert big.numel() > 2 ** 31
    g = P.group_rows(t.repeat(times), 2)
    y = P.linear_typed(big, w, g)
    dx, dw, db = P.linear_typed_backward(big_d, big, w, g, bias=True)
    want_y, want_dx = torch.zeros(block, out, device="cuda"), torch.zeros(block, k, device="cuda")
    for i in range(2):
        of = t == i
        want_y[of], want_dx[of] = x[of].float() @ w[i].float().t(), d[of].float() @ w[i].float()
        assert torch.equal(dw[i], (times * (d[of].float().t() @ x[of].float())).bfloat16())
        assert torch.equal(db[i], times * d[of].float().sum(0))
    for got, want in ((y, want_y), (dx, want_dx)):
        assert bool((got.view(times, block, -1) == want.bfloat16()).all())


def test_weights_beyond_32_bits(torch):
    announce("typed products of 40 types of 8192 x 8192")
    G, dim, n = 40, 8192, 400
    w = _whole(torch, G, dim, dim, seed=5)
    assert w.numel() > 2 ** 31
    x, d = _whole(torch, n, dim, seed=6), _whole(torch, n, dim, seed=7)
    t = torch.arange(n, device="cuda", dtype=torch.int32) % G
    g = P.group_rows(t, G)
    y = P.linear_typed(x, w, g)
    dx, dw, db = P.linear_typed_backward(d, x, w, g, bias=True)
    for i in (0, 31, 32, G - 1):
        of = t == i
        assert torch.equal(y[of], (x[of].float() @ w[i].float().t()).bfloat16())
        assert torch.equal(dx[of], (d[of].float() @ w[i].float()).bfloat16())
        assert torch.equal(dw[i], (d[of].float().t() @ x[of].float()).bfloat16()) and torch.equal(db[i], d[of].float().sum(0))


def test_norm_beyond_32_bits(torch):
    """A row's result does not depend on where it lies."""
    announce("layer norm of 600,000 x 4096")
    times, block, dim = 600, 1000, 4096
    x, r, d = (torch.randn(block, dim, device="cuda").bfloat16() for _ in range(3))
    w, b = torch.randn(dim, device="cuda"), torch.randn(dim, device="cuda")
    y, h, stats = P.layer_norm(x, w, b, residual=r, return_stats=True)
    dx = P.layer_norm_backward(d, h, stats, w, dh=r)[0]
    many = [v.repeat(times, 1) for v in (x, r, d)]
    got = P.layer_norm(many[0], w, b, residual=many[1], return_stats=True)
    got += P.layer_norm_backward(many[2], got[1], got[2], w, dh=many[1])[:1]
    for a, c in zip(got, (y, h, stats, dx)):
        assert bool((a.view(times, *c.shape) == c).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_layer_norm_for_every_set_of_leaves(torch, dtype):
    """The gradients that are asked for are those of the full call, to the bit, with and without the sum's own."""
    announce("layer norm's leaves %s" % dtype)
    n, dim, dt = 70, 100, getattr(torch, dtype)
    x, r, d, dh = (torch.randn(n, dim, device="cuda").to(dt) for _ in range(4))
    w, b = torch.randn(dim, device="cuda"), torch.randn(dim, device="cuda")
    for with_sum in (False, True):
        y, h, stats = P.layer_norm(x, w, b, residual=r, return_stats=True)
        dx, dw, db = P.layer_norm_backward(d, h, stats, w, dh=dh if with_sum else None)
        want = (dx, dx, dw, db)
        for chosen in itertools.product((False, True), repeat=4):
            if not any(chosen):
                continue
            leaves = [v.detach().clone().requires_grad_(c) for v, c in zip((x, r, w, b), chosen)]
            y, h = P.layer_norm(leaves[0], leaves[2], leaves[3], residual=leaves[1])
            asked = [v for v, c in zip(leaves, chosen) if c]
            outs, grads = ((y, h), (d, dh)) if with_sum else ((y,), (d,))
            got = torch.autograd.grad(outs, asked, grads)
            for a, c in zip(got, (v for v, c in zip(want, chosen) if c)):
                assert torch.equal(a, c), chosen
    one = x.clone().requires_grad_()                                    # the same rows twice
    y, _ = P.layer_norm(one, w, b, residual=one)
    _, h, stats = P.layer_norm(x, w, b, residual=x, return_stats=True)
    dx = P.layer_norm_backward(d, h, stats, w)[0]
    assert torch.equal(torch.autograd.grad(y, one, d)[0], dx + dx)
