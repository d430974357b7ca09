"""Table entries outside the pool, among those that a sequence reaches: read as the nearest page."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import SENTINEL, desc, i32, rows
from ig_pages import Pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("entry,nearest", [(-5, 0), (-2 ** 31, 0), (1 << 30, -1), (16, -1)])
@pytest.mark.parametrize("dtype,n_q", [("f16", 1), ("f16", 48), ("f16", 70), ("f32", 1), ("f32", 48)])
def test_read_as_the_nearest_page(ctx, dtype, n_q, entry, nearest):
    B, H, d, N, page = 2, 2, 64, 100, 16
    pages = Pages(B, H, d, 112, page, "i8", 1).fill([N, N], 2)
    n = pages.K.shape[0]
    assert n == 16
    pages.K_scale.nan_to_num_(1.0), pages.V_scale.nan_to_num_(1.0)
    # (the pages that are meant hold what no other does)
    for at, code in ((0, 3), (n - 1, -3)):
        pages.K[at], pages.V[at] = code & 255, 5 * code & 255
    q = rows((B, n_q, H, d), dtype, 3)
    ds = desc(B, H, d, N, 112, dtype, 0.125)
    outs, lists = [], []
    idx, cnt = i32([[0, 33, 40, 47, 99]] * (B * H)), i32([5] * (B * H))
    for e in (entry, nearest % n, 7):
        pages.table[1, 2] = e
        out = torch.full_like(q, SENTINEL)
        sel = [torch.full((B * H, 5, d), SENTINEL, dtype=q.dtype, device="cuda") for _ in "KV"]
        ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, out)
        ctx.ig_gather_pages(ds, pages.struct(), idx, 5, cnt, *sel)
        torch.cuda.synchronize()
        outs.append(out)
        lists.append(sel)
    assert torch.equal(outs[0], outs[1]) and not torch.equal(outs[1][1], outs[2][1]) and torch.equal(outs[1][0], outs[2][0])
    for a, b, c in zip(*lists):
        assert torch.equal(a, b) and not torch.equal(b, c)
