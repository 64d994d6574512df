"""Layer norm's gradients of rows whose numbers, or what they are multiplied with, are very large or very small."""
import numpy as np
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu
from oracle import layer as O
from test_gpu_layer import DTYPES, ROUND, UNIT, _check_norm, _host, _up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [1, 3, 31, 100, 128, 300, 700, 768, 1100, 1500, 3000, 5000, 9000])
def test_rows_of_one_large_number(torch, dim, dtype):
    """Distances are zeros and 1/sqrt(eps) is large: a mean times that is beyond float32, and of no matter."""
    announce("layer norm of rows of one large number, %d %s" % (dim, dtype))
    rng = np.random.default_rng(dim)
    h = rng.standard_normal((9, dim))
    for row, v in enumerate((1e25, -1e25, 3e20, 1e29, -1e29, 1e30)):
        h[row] = v
    x, d = _up(torch, h, dtype)[0], _up(torch, rng.standard_normal((9, dim)), dtype)[0]
    w, b = (_up(torch, rng.standard_normal(dim))[0] for _ in range(2))
    for eps in (1e-30, 1e-35):
        _check_norm(torch, dtype, x, None, None, None, d, None, eps=eps)
        _check_norm(torch, dtype, x, None, w, b, d, d, eps=eps)


def _gradients(rng, kind, n, dim):
    """x, dy, weights, dh: gradients or their products with the weights near the end of float32 or beyond it, whose own gradient is not."""
    x, dy, w, dh = 4 * rng.standard_normal((n, dim)), rng.uniform(-3e38, 3e38, (n, dim)), None, None
    if kind == "one sign":
        dy = np.abs(dy)
    if kind == "products":
        x, dy, w = 1e4 * x, 1e30 * rng.standard_normal((n, dim)), 1e10 * rng.standard_normal(dim)
    if kind == "a mean":                    # large in one lane, small in the others, which subtract its mean
        dy = rng.standard_normal((n, dim))
        dy[:, :4] = 3e38
    if kind == "two gradients":             # dx alone leaves float32, with dh it does not
        x, dy, dh = 0.0625 * x, np.zeros((n, dim)), np.zeros((n, dim))
        dy[:, 0], dh[:, 0] = 1.2e38, -3e38
    return x, dy, w, dh


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 100, 300, 768, 1500, 4100, 9000])
@pytest.mark.parametrize("kind", ["signs", "one sign", "products", "a mean", "two gradients"])
def test_large_gradients(torch, kind, dim, dtype):
    """Sums and products on the way may leave float32's range; the gradient does not."""
    announce("layer norm of large gradients, %s %d %s" % (kind, dim, dtype))
    rng = np.random.default_rng(dim)
    x, dy, w, dh = _gradients(rng, kind, 9, dim)
    x, dy, dh = (None if v is None else _up(torch, v, dtype)[0] for v in (x, dy, dh))
    w = None if w is None else _up(torch, w)[0]
    _, stats = P.layer_norm(x, w, return_stats=True)
    dx = P.layer_norm_backward(dy, x, stats, w, dh=dh)[0]
    _, _, rstd, xh = O.layer_norm(_host(x), eps=np.float64(np.float32(1e-5)))
    want = O.layer_norm_backward(_host(dy), _host(x), None if w is None else _host(w), np.float64(np.float32(1e-5)))[0]
    if dh is not None:
        assert (np.abs(want[:, 0]) > 3.41e38).any()
        want = want + _host(dh)
    assert np.abs(want).max() < 3.3e38
    # the bound of _check_norm, which is relative
    g = np.abs(_host(dy) * (1 if w is None else _host(w)))
    size = (40 * g.mean(1, keepdims=True) + 6 * g + 48 * np.abs(xh) * (g * np.abs(xh)).mean(1, keepdims=True)) * rstd[:, None]
    tol = UNIT / 2 * (size + 2 * np.abs(want))
    assert (np.abs(_host(dx) - want) <= tol + ROUND[dtype] * (np.abs(want) + tol) + 1e-37).all()
