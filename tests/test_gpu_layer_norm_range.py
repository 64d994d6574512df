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
