"""The serving example: its layer against the operators' definitions."""
import math
import os
import sys

import numpy as np
import pytest

from gpu_util import announce, require_gpu
from oracle import layer8 as O

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_example_serves_what_its_caches_hold():
    torch = require_gpu()
    import paper_2203_14883_amd as P
    import serve_attention as S
    announce("serving example")
    layer, last = S.serve(edges=8000, batches=6, batch=200, dtype=torch.float32)
    assert last["out"].shape == (400, S.DIM) and torch.isfinite(last["out"]).all()
    assert int(layer.length.max()) >= 2
    # the last state once more: attention over slots and over histories, by definition
    roots, times = last["roots"][:40], last["times"][:40]
    rows = last["memory"][roots.long()]
    q, _, _, _ = layer.project(rows)
    hop = P.sample(last["graph"], roots, times, (S.FANOUT,), "recent")[0]
    slots = hop.nbr.view(-1, S.FANOUT)
    assert (slots < 0).any() and (slots >= 0).any()
    scale = 1 / math.sqrt(S.HEAD)
    host = lambda c: O.Cache(c.data.cpu().numpy(), c.scales.cpu().numpy(), c.dim)  # noqa: E731
    qh = q.cpu().numpy()[:, None]
    nodes, hist = host(layer.nodes), host(layer.history)
    near, _ = nodes.attend(qh, slots.cpu().numpy(), None, None, scale)
    end = layer.length[roots.long()].cpu().numpy()
    past, _ = hist.attend(qh, layer.table[roots.long()].cpu().numpy(), np.maximum(end - S.WINDOW, 0), end, scale)
    got = P.cache_attend(layer.nodes, q, slots).cpu().numpy()
    # float32: 2^-20 of the largest value for the weights, as much for the scores' rounding
    tol = 4 * 2.0 ** -20 * 127 * max(nodes.scales.max(), hist.scales.max()) * (1 + np.abs(qh).max() * 127 * nodes.scales.max())
    assert np.abs(got - near[:, 0]).max() <= tol
    out = layer.attend(last["graph"], roots, times, rows)
    both = (near + past).reshape(40, -1).astype(np.float32)
    q8, s8, _ = O.norm_quant(both, None, None, 0.0, normalize=False)
    want = O.linear_i8(q8, s8, layer.out[0].cpu().numpy(), layer.out[1].cpu().numpy(), None)
    # a sum near a rounding boundary may give the next byte: one step of each of a row's bytes at most
    step = s8[:, None] * (np.abs(layer.out[0].cpu().numpy().astype(np.float64)) * layer.out[1].cpu().numpy()[:, None]).sum(1)[None]
    assert np.all(np.abs(out.cpu().numpy() - want) <= step)
    assert np.abs(out.cpu().numpy() - want).mean() <= 0.02 * np.abs(want).mean()
