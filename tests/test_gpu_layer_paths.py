"""Groups that make no sense, at the sizes of every kernel of the typed products: nothing outside the outputs and the
workspace is written, and rows that no place names keep what they held."""
import ctypes as C

import pytest

import paper_2203_14883_amd as P
from gpu_util import announce, require_gpu
from paper_2203_14883_amd import binding as B
from test_gpu_layer import _type

pytestmark = pytest.mark.gpu
GUARD = 4096            # bytes on each side


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


class Guarded:
    """Memory of `size` bytes between two stretches that must keep their bytes."""

    def __init__(self, torch, size):
        self.all = torch.full((size + 2 * GUARD,), 0x5a, device="cuda", dtype=torch.uint8)
        self.inner = self.all[GUARD:GUARD + size]
        self.ptr = self.inner.data_ptr()

    def kept(self):
        return bool((self.all[:GUARD] == 0x5a).all()) and bool((self.all[-GUARD:] == 0x5a).all())


# rows, in, out, types of element: tiles of 16, 64, 128 and 256, straight to LDS and through registers
SIZES = [(100, 64, 64, "f32"), (5000, 64, 512, "f32"), (5000, 67, 515, "f32"), (3000, 136, 128, "bf16"), (3001, 135, 129, "bf16"),
         (20_000, 72, 256, "bf16"), (20_000, 256, 768, "bf16"), (20_000, 261, 771, "bf16")]
G = 5


def offsets_of(n):
    yield [0, n // 2, n, 10 ** 12, 10 ** 15, 2 ** 62]                   # beyond the rows
    yield [0, -7, n // 2, -2 ** 62, n - 10, n]                          # below them
    yield [0, n, 0, n, 0, n]                                            # three types of all rows: more parts than there is room for
    yield [9, n, n // 3, n - 1, 2, n // 2]                              # types that overlap, rows of no type that have one
    yield [0, n, n, n, n, 0]


@pytest.mark.parametrize("ordered", [True, False])
@pytest.mark.parametrize("n,k,out,dtype", SIZES)
def test_groups_that_make_no_sense(torch, n, k, out, dtype, ordered):
    announce("groups that make no sense, %d x %d -> %d %s %s" % (n, k, out, dtype, ordered))
    t, e, dt = _type(torch, dtype), 4 if dtype == "f32" else 2, B.OUT_F32 if dtype == "f32" else B.OUT_BF16
    x, d, w = (torch.randn(*s, device="cuda").to(t) for s in ((n, k), (n, out), (G, out, k)))
    bias = torch.randn(G, out, device="cuda")
    order = torch.arange(n, dtype=torch.int32, device="cuda")
    order[::7], order[3::7] = 2 ** 31 - 1, -5
    unnamed = torch.zeros(n, dtype=torch.bool, device="cuda")
    if ordered:
        unnamed[::7] = unnamed[3::7] = True
    weights = B.c_typed_weights(w.data_ptr(), out * k, k, out, k)
    L, stream = P.lib(), torch.cuda.current_stream().cuda_stream
    for offsets in offsets_of(n):
        at = torch.tensor(offsets, dtype=torch.int64, device="cuda")
        g = B.c_row_groups(order.data_ptr() if ordered else None, at.data_ptr(), n, G, 0)
        need = L.tgl_linear_typed_grad_w_workspace(C.byref(g), out, k, dt)
        y, dx, dw, db, ws = (Guarded(torch, s) for s in (n * out * e, n * k * e, G * out * k * e, G * out * 4, need))
        assert L.tgl_linear_typed(C.byref(g), x.data_ptr(), k, C.byref(weights), bias.data_ptr(), y.ptr, out, dt, stream) == 0
        assert L.tgl_linear_typed_grad_x(C.byref(g), d.data_ptr(), out, C.byref(weights), dx.ptr, k, dt, stream) == 0
        assert L.tgl_linear_typed_grad_w(C.byref(g), d.data_ptr(), out, x.data_ptr(), k, out, k, dw.ptr, db.ptr, dt,
                                         ws.ptr if need else None, need, stream) == 0
        torch.cuda.synchronize()
        assert all(v.kept() for v in (y, dx, dw, db, ws)), offsets
        for v, columns in ((y, out), (dx, k)):
            assert bool((v.inner.view(n, columns * e)[unnamed] == 0x5a).all()), offsets
