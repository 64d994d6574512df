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
