"""Appends to pages whose rows are more than one launch takes: refused for their size, before anything is launched."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import desc
from ig_pages import Pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


# A launch takes 2^32 - 1 threads.  Keys and values: a workgroup each for every page that the new rows of a sequence can touch, of a
# thread for 32 channels of a page's new rows, at least 64; queries: a thread for 16 channels of a row.  (One head each: no heads in turn.)
@pytest.mark.parametrize("B,d,n_rows,group,page,queries,code", [
    (7400000, 256, 9, 1, 16, True, ig.IG_ESHAPE),            # 2 x 2 pages x 128 threads, and 144 for queries: 656 a sequence
    (6500000, 256, 9, 1, 16, True, ig.IG_EINVAL),            # 2^31.99
    (7400000, 256, 9, 1, 16, False, ig.IG_EINVAL),           # 512 a sequence: 2^31.8
    (16760784, 32, 2, 1, 16, False, ig.IG_EINVAL),           # the most sequences of one slot that a call takes; 2 x 2 x 64 each: 2^31.998
    (16760784, 256, 1, 4, 16, True, ig.IG_EINVAL),           # 2 x 64, and 16 for queries (four heads in turn): 2^31.2
])
def test_more_rows_than_a_launch_takes(ctx, B, d, n_rows, group, page, queries, code):
    """(Every call has an unaligned array, which is refused later: nothing is launched or read.)"""
    p = Pages(1, 1, d, page, page, "i8", 1)
    x = torch.zeros(1 << 12, dtype=torch.float16, device="cuda")
    bad = x.data_ptr() + 2
    with pytest.raises(ig.IgError) as e:
        ctx.ig_append_pages(desc(B, 1, d, 1, 1, "f16"), p.struct(n_pages=1), None, group, n_rows, x if queries else None, bad, x, 0,
                            None, None, None, x if queries else None)
    assert e.value.code == code, e.value
