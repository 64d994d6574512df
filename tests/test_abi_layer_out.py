"""An output that shares memory with an input is refused before anything is enqueued: other workgroups still read it."""
import pytest
import torch

import paper_2203_14883_amd as P
from paper_2203_14883_amd import layer


@pytest.fixture
def on_host(monkeypatch):
    """The calls' checks of host tensors, up to the library."""
    class Reached(Exception):
        pass

    def reached():
        raise Reached

    monkeypatch.setattr(layer, "_device", lambda t, name: -1)
    monkeypatch.setattr(layer, "_raw_stream", lambda stream, dev: None)
    monkeypatch.setattr(layer, "lib", reached)
    return Reached


def _groups(n, types=2):
    return P.RowGroups(torch.zeros(types + 1, dtype=torch.int64), torch.zeros(n, dtype=torch.int32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_linear_typed_refuses_inputs_as_output(on_host, dtype):
    n, k = 9, 16
    x, w, g = torch.zeros(n, k, dtype=dtype), torch.zeros(2, k, k, dtype=dtype), _groups(n)
    both = torch.zeros(n + 3, k, dtype=dtype)
    beside = torch.zeros(n, 2 * k, dtype=dtype)
    for a, out in ((x, x), (x, x.view(n, k)), (both[:n], both[3:]), (both[3:], both[:n]), (both[:1].expand(n, k), both[:n]),
                   (beside[:, :k], beside[:, 1:k + 1]), (beside[:, 2:k + 2], beside[:, :k])):
        with pytest.raises(ValueError, match="out shares memory with x"):
            P.linear_typed(a, w, g, out=out)
    few = _groups(2 * k)
    with pytest.raises(ValueError, match="out shares memory with w"):
        P.linear_typed(torch.zeros(2 * k, k, dtype=dtype), w, few, out=w.view(2 * k, k))
    if dtype == torch.float32:
        b = torch.zeros(2, k)
        with pytest.raises(ValueError, match="out shares memory with bias"):
            P.linear_typed(torch.zeros(2, k), w, _groups(2), b, out=b)
        place = torch.zeros(8, dtype=torch.int32)
        with pytest.raises(ValueError, match="out shares memory with the groups"):
            P.linear_typed(torch.zeros(8, 1), torch.zeros(2, 1, 1), P.RowGroups(torch.zeros(3, dtype=torch.int64), place),
                           out=place.view(torch.float32).view(8, 1))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_linear_typed_takes_outputs_beside_inputs(on_host, dtype):
    """Columns beside the input's, every other row, rows behind it, one row, none: nothing is shared."""
    n, k = 9, 16
    w, g = torch.zeros(2, k, k, dtype=dtype), _groups(n)
    beside, rows = torch.zeros(n, 2 * k + 3, dtype=dtype), torch.zeros(2 * n, k, dtype=dtype)
    square = torch.zeros(n, k, dtype=dtype)
    for x, out in ((beside[:, :k], beside[:, k:2 * k]), (beside[:, k + 3:], beside[:, 1:k + 1]), (rows[::2], rows[1::2]), (rows[1::2], rows[::2]),
                   (rows[:n], rows[n:]), (rows[n:], rows[:n]), (square, torch.zeros(n, k, dtype=dtype))):
        with pytest.raises(on_host):
            P.linear_typed(x, w, g, out=out)
    with pytest.raises(on_host):
        P.linear_typed(rows[:1], w, _groups(1), out=rows[1:2])
    with pytest.raises(on_host):
        P.linear_typed(rows[:0], w, _groups(0), out=rows[:0])
    # weights between an output's columns
    wide = torch.zeros(2, k, 2 * k, dtype=dtype)
    with pytest.raises(on_host):
        P.linear_typed(torch.zeros(2 * k, k, dtype=dtype), wide[:, :, :k], _groups(2 * k), out=wide.view(2 * k, 2 * k)[:, k:])


def test_shared_memory_is_found_by_counting():
    """Against the sets of elements: nothing that shares one is taken, and nothing of the same distance that shares none is refused."""
    import random
    rng = random.Random(3)
    taken = refused = 0
    for _ in range(4000):
        store = torch.zeros(200)
        pitch = rng.randint(1, 12)

        def piece(step):
            n, k = rng.randint(1, 6), rng.randint(1, step)
            return store.as_strided((n, k), (step, 1), rng.randint(0, 60)), (n, k, step)

        (a, (an, ak, astep)), (b, (bn, bk, bstep)) = piece(pitch), piece(rng.choice([pitch, rng.randint(1, 12)]))
        sets = [{t.storage_offset() + i * step + j for i in range(n) for j in range(k)}
                for t, n, k, step in ((a, an, ak, astep), (b, bn, bk, bstep))]
        try:
            layer._separate(a, (b, "b"))
            ok = True
        except ValueError:
            ok = False
        if sets[0] & sets[1]:
            assert not ok
            refused += 1
        else:
            assert ok or astep != bstep
            taken += ok
    assert taken > 500 and refused > 500
