"""The calls over a whole pool without a context: refused before anything is looked at, through both marshallings."""
import pytest

import paper_2406_19707_amd as ig
from paper_2406_19707_amd import binding

COUNTS = {"ig_cache_attention": 12, "ig_tree_attention": 14, "ig_append_rows": 16, "ig_pool_evict": 12}


@pytest.mark.parametrize("name", COUNTS)
def test_no_context(name):
    d = ig.IgDesc(B=1, H=1, d=64, r=1, N=8)
    numbers = {"ig_cache_attention": 2, "ig_tree_attention": 2, "ig_append_rows": 1, "ig_pool_evict": 1}[name]
    args = [None, d] + [1] * numbers + [None] * (COUNTS[name] - 2 - numbers)
    assert len(getattr(binding.lib(), name).argtypes) == COUNTS[name]
    assert binding._through_ctypes(name, *args) == ig.IG_EINVAL
    assert getattr(binding._Entries(), name)(*args) == ig.IG_EINVAL


def test_reserve_without_context():
    assert ig.lib().ig_reserve_cache(None, None, 1, 1) == ig.IG_EINVAL
