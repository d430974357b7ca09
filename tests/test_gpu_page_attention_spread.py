"""Attention over pages whose scales of V lie further apart than the exponents of a float32 reach: a slot's share of the softmax's sum
does not depend on its page's scale of V."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import SENTINEL, desc, rows
from ig_pages import LEAST, Pages, check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def attend(ctx, pages, n, n_q, dtype, scale=0.125):
    B, H, d, N_cap = pages.shape
    q = rows((B, n_q, H, d), dtype, 3)
    out = torch.full_like(q, SENTINEL)
    ctx.ig_page_attention(desc(B, H, d, n, N_cap, dtype, scale), pages.struct(), 1, n_q, q, None, None, out)
    torch.cuda.synchronize()
    check_attention(pages, q, [n] * B, [n_q] * B, 1, scale, dtype, out, out)


def zero_values(pages, at):
    """as ig_append_pages stores them"""
    pages.V[at], pages.V_scale[at] = 0, LEAST


@pytest.mark.parametrize("top", [40, 62, 100, 119])
@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("which", ["every second page zero", "the first page large", "the last page large"])
def test_large_values_beside_zeros(ctx, which, n_q, top):
    """Within a tile, among the tiles of a wave, and among waves."""
    N, page = 297, 16
    pages = Pages(1, 2, 64, N, page, "i8", 1).fill([N], 2, spread=0)
    at = pages.table[0].long()
    pages.V_scale[at] = 2.0 ** top
    zero_values(pages, {"every second page zero": at[1::2], "the first page large": at[1:], "the last page large": at[:-1]}[which])
    attend(ctx, pages, N, n_q, "f32")


@pytest.mark.parametrize("n_q", [1, 20])
@pytest.mark.parametrize("large", [0, 70, 155])
def test_among_slices(ctx, large, n_q):
    N, page = 10000, 64
    pages = Pages(1, 1, 128, N, page, "e4m3", 1).fill([N], 2, spread=0)
    at = pages.table[0].long()
    pages.V_scale[at] = 2.0 ** 90
    zero_values(pages, torch.cat([at[:large], at[large + 1:]]))
    attend(ctx, pages, N, n_q, "f32", 0.01)


@pytest.mark.parametrize("n_q", [1, 70])
def test_logits_apart_as_well(ctx, n_q):
    """Large values at small weights beside small values at large ones, and the other way round."""
    N, page = 200, 16
    for k_large in (0.03125, 4.0):
        pages = Pages(1, 2, 64, N, page, "i8", 1).fill([N], 2, spread=0)
        at = pages.table[0].long()
        pages.V_scale[at[::2]], pages.V_scale[at[1::2]] = 2.0 ** 70, 2.0 ** -75
        pages.K_scale[at[::2]] = k_large
        attend(ctx, pages, N, n_q, "f32")


@pytest.mark.parametrize("n_q", [1, 70])
def test_half_precision(ctx, n_q):
    """The spread that half rows can have, and a float32 cache's zeros beside it."""
    N, page = 200, 16
    pages = Pages(1, 2, 64, N, page, "i8", 1).fill([N], 2, spread=0)
    at = pages.table[0].long()
    pages.V_scale[at] = 2.0 ** 9
    zero_values(pages, at[1::2])
    attend(ctx, pages, N, n_q, "f16")
