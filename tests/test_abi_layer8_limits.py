"""What the 8-bit operators refuse because no launch could take it (host checks only)."""
from paper_2203_14883_amd import binding as B
from test_abi_layer8 import _attend, _cache, _seqs


def test_attend_refuses_a_sequence_of_more_tiles_than_a_launch_has():
    """2^10 heads of 2^20 queries: 2^25 workgroups of 256 threads for one sequence."""
    cache = _cache(heads=1024, dim=16)
    assert _attend(cache=cache, seqs=_seqs(seqs=1), heads=1024, queries=1 << 20, t=1 << 14, h=16) == B.EINVAL
