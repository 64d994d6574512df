"""Sums over rows, on whole numbers: what float32 holds without rounding has to be right to the bit, so no row can be
missing or counted twice, and what it does not hold is the nearest number to the sum."""
import numpy as np
import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu
from oracle import layer as O
from test_gpu_layer import DTYPES, _host, _type

pytestmark = pytest.mark.gpu

# rows, in, out, types, empty: every tile of the weights' gradient, with loads straight to LDS and through registers, types that
# are cut into many parts, a few, none, that are not there
CASES = [(50_000, 256, 512, 6, 0.02), (42_000, 264, 328, 3, 0.1), (20_001, 261, 515, 2, 0.0), (9000, 128, 256, 1, 0.0), (9001, 100, 200, 3, 0.1),
         (9001, 101, 203, 3, 0.1), (33_000, 67, 45, 2, 0.0), (40_000, 200, 264, 200, 0.0), (70_000, 48, 33, 3, 0.9), (20_000, 64, 72, 40, 0.3),
         (16_384, 1024, 1280, 2, 0.0), (257, 40, 72, 2, 0.1), (513, 200, 264, 1, 0.0)]


def whole_numbers(n, k, out, G, empty):
    """Types of rows, rows, weights, biases and gradients, all whole numbers from -3 to 3: a product is 9 at most, and sums of
    1.8 million of them are exact in float32."""
    rng = np.random.default_rng(n + k + out)
    t = np.minimum(rng.geometric(0.5, n) - 1, G - 1)        # some types have many rows, others few or none
    t = (t * 37 + 3) % G
    t[rng.random(n) < empty] = -1
    return (t,) + tuple(rng.integers(-3, 4, s).astype(np.float32) for s in ((n, k), (G, out, k), (G, out), (n, out)))


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


def _rounded(torch, a, dtype):
    return torch.from_numpy(a).to(torch.float32).to(_type(torch, dtype)).cuda()      # exact, then to nearest


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k,out,G,empty", CASES)
def test_whole_numbers(torch, n, k, out, G, empty, dtype):
    announce("whole numbers %d x %d -> %d, %d types, %s" % (n, k, out, G, dtype))
    t, x, w, b, d = whole_numbers(n, k, out, G, empty)
    g = P.group_rows(torch.from_numpy(t.astype(np.int32)).cuda(), G)
    up = lambda a: torch.from_numpy(a).to(_type(torch, dtype)).cuda()
    y = P.linear_typed(up(x), up(w), g, torch.from_numpy(b).cuda())
    dx, dw, db = P.linear_typed_backward(up(d), up(x), up(w), g, bias=True)
    want = np.zeros((n, out))
    for i in range(G):
        want[t == i] = x[t == i].astype(np.float64) @ w[i].T.astype(np.float64) + b[i]
    wx, ww, wb = O.linear_backward(d, x, w, t)
    assert max(np.abs(v).max() for v in (want, wx, ww, wb)) < 2 ** 24
    assert torch.equal(y, _rounded(torch, want, dtype)) and torch.equal(dx, _rounded(torch, wx, dtype))
    assert torch.equal(dw, _rounded(torch, ww, dtype)) and torch.equal(db, _rounded(torch, wb, "f32"))


@pytest.mark.parametrize("n,k,out,dtype", [(65_537, 2560, 4096, "f32"), (1_000_003, 64, 64, "f32"), (3_000_001, 16, 16, "f32"), (132_001, 768, 1024, "bf16"),
                                           (140_000, 200, 264, "bf16"), (1_000_003, 96, 96, "bf16"), (3_000_001, 16, 16, "bf16"), (400_000, 33, 45, "bf16")])
def test_biases_gradients_are_the_nearest_numbers(torch, n, k, out, dtype):
    """Odd numbers of 20 bits (8 in bfloat16), whose sums float32 does not hold: eight of them together it does, and from
    there on sums have 64 bits, so the result is rounded once.  The rows are one, n times."""
    announce("biases' gradients, %d rows %s" % (n, dtype))
    rng = np.random.default_rng(n + k)
    v = 2 * rng.integers(2 ** 18, 2 ** 19, (1, out)) + 1 if dtype == "f32" else 2 * rng.integers(64, 128, (1, out)) + 1
    v *= rng.choice([-1, 1], (1, out))
    d = torch.from_numpy(v.astype(np.float32)).to(_type(torch, dtype)).cuda()
    x = torch.ones(1, k, device="cuda", dtype=d.dtype)
    g = P.RowGroups(torch.tensor([0, 3, n], device="cuda"))
    w = torch.zeros(1, out, k, device="cuda", dtype=d.dtype).expand(2, out, k)
    db = P.linear_typed_backward(d.expand(n, out), x.expand(n, k), w, g, bias=True)[2]
    want = np.concatenate([3 * v, (n - 3) * v])
    assert np.array_equal(_host(db), want.astype(np.float32).astype(np.float64))


def test_parts_of_weights_gradients_are_joined_in_64_bits(torch):
    """Each stretch's sum is exact in float32, the sum of all is not: it is the number nearest to it."""
    announce("weights' gradients of many parts")
    n, k, out = 3_000_001, 16, 16
    x, d = (torch.randint(1, 8, (n, c), device="cuda", generator=torch.Generator("cuda").manual_seed(c + i)).float() for i, c in enumerate((k, out)))
    dw, db = P.linear_typed_backward(d, x, torch.zeros(1, out, k, device="cuda"), P.RowGroups(torch.tensor([0, n], device="cuda")), bias=True)[1:]
    want = torch.zeros(out, k, device="cuda", dtype=torch.float64)
    for a, c in zip(d.split(500_000), x.split(500_000)):
        want += a.double().t().contiguous() @ c.double()
    assert float(want.min()) > 2 ** 24 and 49 * n / 2000 < 2 ** 24      # there are 2560 stretches of even length
    assert torch.equal(dw[0], want.float()) and torch.equal(db[0], d.double().sum(0).float())
