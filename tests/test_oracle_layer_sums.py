"""The whole numbers that the weights' gradients are tested on show a lost row: planted in the oracle, on the CPU."""
import numpy as np
import pytest
import torch

from test_gpu_layer_sums import CASES, whole_numbers


@pytest.mark.parametrize("n,k,out,G,empty", CASES)
def test_lost_rows_are_seen(n, k, out, G, empty):
    t, x, _, _, d = whole_numbers(n, k, out, G, empty)
    for rows in {len(np.flatnonzero(t == g)): np.flatnonzero(t == g) for g in range(G)}.values():
        if not len(rows):
            continue
        dw = d[rows].T.astype(np.float64) @ x[rows]
        for lost in (rows[-1:], rows[:256], rows[len(rows) // 2:][:16]):        # the last row, a stretch, a few of a step
            less = dw - d[lost].T.astype(np.float64) @ x[lost]
            for dtype in (torch.float32, torch.bfloat16):
                assert not torch.equal(torch.from_numpy(dw).to(dtype), torch.from_numpy(less).to(dtype))
            assert d[lost].sum(0).any()
