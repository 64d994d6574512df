"""Rows and products in 8 bits at the ends of their number ranges."""
import math

import numpy as np
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu
from oracle import layer8 as O
from test_gpu_layer8 import HALF, TYPES, _up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [5, 64, 700, 1500, 3000, 8200])
@pytest.mark.parametrize("size,eps", [(1e19, 1e-6), (1e20, 1e-6), (1e30, 0.0), (2e37, 1e-6), (1e-20, 0.0), (1e-25, 0.0), (1e-22, 1e-40), (1e-3, 0.0)])
def test_norm_of_rows_of_any_size(size, eps, dim, dtype):
    """h / rms(h) is near 1 however large or small h is: neither squares nor their mean leave the range."""
    torch = require_gpu()
    announce("norm of rows near %g, dim %d %s" % (size, dim, dtype))
    rng = np.random.default_rng(dim)
    x, xh = _up(torch, size * rng.standard_normal((3, dim)), dtype)
    r, rh = _up(torch, size * rng.standard_normal((3, dim)), dtype)
    w, wh = _up(torch, 1 + 0.1 * rng.standard_normal(dim))
    q, scale, h = P.norm_quant(x, w, residual=r, eps=eps)
    oq, oscale, _ = O.norm_quant(xh, rh, wh, float(np.float32(eps)))
    assert np.array_equal(q.cpu().numpy(), oq)
    np.testing.assert_allclose(scale.cpu().numpy(), oscale, rtol=(dim / 64 + 24) * HALF)
    # the bytes come from float32 operations, the step from one: rows that are a norm's
    got = oq * scale.cpu().numpy()[:, None].astype(np.float64)
    if eps == 0 or size > 1:
        rms = np.sqrt(np.mean((got / wh) ** 2, 1))
        assert np.all(np.abs(rms - 1) <= 0.05)


@pytest.mark.parametrize("m", [1, 20, 300])
@pytest.mark.parametrize("k", [131071, 131072])
def test_linear_i8_of_the_smallest_bytes(k, m):
    """Sums of (-128)^2 reach 2^31 at the largest k."""
    torch = require_gpu()
    announce("linear_i8 of -128, %d rows, k %d" % (m, k))
    x = torch.full((m, O.round16(k)), -128, dtype=torch.int8).cuda()[:, :k]
    w = torch.full((900, O.round16(k)), -128, dtype=torch.int8).cuda()[:, :k]
    w[1] = 127
    w[2, ::2] = 127
    y = P.linear_i8(x, torch.ones(m).cuda(), w, torch.ones(900).cuda(), out_dtype=torch.float32).double()
    for j, total in ((0, 128 * 128 * k), (1, -128 * 127 * k), (2, 128 * 128 * (k // 2) - 128 * 127 * (k - k // 2))):
        assert (y[:, j] - float(total)).abs().max() <= abs(total) * 2.0 ** -24
