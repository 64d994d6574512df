"""HistoryCache as a Python object; tensors that carry derivatives."""
import copy
import pickle

import pytest
import torch
import torch.autograd.forward_ad as fwd

import paper_2203_14883_amd as P
from paper_2203_14883_amd import layer8


@pytest.mark.parametrize("how", ["copy", "pickle"])
def test_history_cache_can_be_copied(how):
    """A copy has its own tensors and a view of those."""
    c = P.HistoryCache.empty(6, 2, 50, 4, device="cpu")
    c.data[3, 1, 0, 2, 7] = 9
    c.scales[3] = 0.5
    d = copy.deepcopy(c) if how == "copy" else pickle.loads(pickle.dumps(c))
    assert torch.equal(c.data, d.data) and torch.equal(c.scales, d.scales) and d.dim == 50
    assert d.data.data_ptr() != c.data.data_ptr()
    v = d.c_view()
    assert (v.data, v.scales, v.num_pages, v.page_tokens, v.heads, v.dim) == (d.data.data_ptr(), d.scales.data_ptr(), 6, 4, 2, 50)
    both = copy.deepcopy([c, c.data])
    assert both[0].data is both[1]


def test_tensors_with_a_tangent_are_refused():
    """A forward-mode derivative would be lost in silence: it is refused as a reverse-mode one is, before anything else."""
    x = torch.randn(4, 32)
    with fwd.dual_level():
        dual = fwd.make_dual(x, torch.ones_like(x))
        for f in (lambda: layer8._also(dual, "q", -1), lambda: layer8._vector(dual[0], 32, "weight", -1)):
            with pytest.raises(ValueError, match="gradient"):
                f()
        layer8._also(x, "q", -1)            # one without is taken
        layer8._also(fwd.unpack_dual(dual).primal, "q", -1)
        with pytest.raises(ValueError):
            P.norm_quant(dual)
    layer8._also(x, "q", -1)
