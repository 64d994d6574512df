"""The training example: it runs, and its gradients are those of the same layer in 64 bits."""
import os
import sys

import pytest

from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _typed(x, w, kind, bias=None):
    """Rows times their kind's weights, kind by kind; zeros for kind -1."""
    y = x.new_zeros(len(x), w.shape[1])
    for k in range(len(w)):
        rows = (kind == k).nonzero()[:, 0]
        y = y.index_add(0, rows, x[rows] @ w[k].T + (0 if bias is None else bias[k]))
    return y


def test_example_trains_with_the_layers_gradients():
    torch = require_gpu()
    import train_typed as S
    announce("training example")
    layer, last = S.train(batches=3, batch=200, edges=8000, nodes=700)
    assert len(last["losses"]) == 3 and all(map(torch.isfinite, map(torch.tensor, last["losses"])))
    got = torch.autograd.grad(S.loss_of(layer, last["rows"], last["kind"], last["src"], last["dst"], last["slots"]), layer.parameters)
    # the same in 64 bits, by torch's operators
    own, near, bias, gamma, beta = wide = [p.detach().double().requires_grad_() for p in layer.parameters]
    rows, kind, slots = last["rows"].double(), last["kind"], last["slots"]
    roots = torch.cat([last["src"], last["dst"]]).long()
    assert (slots < 0).any()

    class Wide:
        def __call__(self, rows, kind, roots, slots):
            flat = slots.reshape(-1).long()
            y = _typed(rows[flat.clamp(min=0)], near, torch.where(flat < 0, -1, kind[flat.clamp(min=0)]))
            y = y.view(len(slots), S.FANOUT, -1).sum(1) / (slots >= 0).sum(1, keepdim=True).clamp(min=1)
            h = y + _typed(rows[roots.long()], own, kind[roots.long()], bias)
            c = h - h.mean(1, keepdim=True)
            return c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma + beta

    want = torch.autograd.grad(S.loss_of(Wide(), rows, kind, last["src"], last["dst"], slots), wide)
    for a, b in zip(got, want):
        # float32: each of the step's dozen operations is off by a few 2^-24 of what it adds up; sums over 400 roots, 64
        # columns and 10 slots of either sign keep that below 2^-24 * 12 * 64 of the largest gradient
        assert float((a.double() - b).abs().max()) <= 12 * 64 * 2.0 ** -24 * float(b.abs().max())
