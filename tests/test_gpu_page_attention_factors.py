"""Attention over pages where the factor of the logits, K's scale times the queries' and the logits' own, leaves the range of a float:
a masked slot has no weight whatever it is, and keys of zero have logits of zero."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import SENTINEL, desc, i32, rows
from ig_pages import LEAST, Pages, check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def attend(ctx, pages, q, kv, dtype, scale):
    B, H, d, N_cap = pages.shape
    n_q = q.shape[1]
    out = torch.full_like(q, SENTINEL)
    before = out.clone()
    ctx.ig_page_attention(desc(B, H, d, max(kv), N_cap, dtype, scale), pages.struct(), 1, n_q, q, None, i32(kv), out)
    torch.cuda.synchronize()
    check_attention(pages, q, kv, [n_q] * B, 1, scale, dtype, out, before)
    return out


@pytest.mark.parametrize("queries", ["zero", "tiny", "a zero row among others"])
@pytest.mark.parametrize("n_q", [1, 40, 70])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_keys_of_zero(ctx, dtype, d, n_q, queries):
    """Zero keys as ig_append_pages stores them, i.e. with the smallest scale: every query's weights are alike, and its row is the
    mean of the values that it sees."""
    B, H, kv = 2, 2, [77, 301]
    pages = Pages(B, H, d, 320, 32, "i8", 1)
    k = torch.zeros((B, 301, H, d), dtype=torch.float16 if dtype == "f16" else torch.float32, device="cuda")
    v = rows((B, 301, H, d), dtype, 2)
    ctx.ig_append_pages(desc(B, H, d, 0, 320, dtype), pages.struct(), None, 1, 301, None, k, v, 0, i32(kv), i32([0, 0]), None, None)
    assert (pages.K_scale[pages.table[1, :10].long()] == LEAST).all()
    q = rows((B, n_q, H, d), dtype, 3)
    if queries == "zero":
        q.zero_()
    elif queries == "tiny":
        q *= 2.0 ** -20 if dtype == "f16" else 2.0 ** -90
    else:
        q[:, ::3] = 0
    attend(ctx, pages, q, kv, dtype, 0.125)


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -100, -2.0 ** -126])
@pytest.mark.parametrize("n_q", [1, 40, 70])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_small_scales_of_the_logits(ctx, dtype, n_q, scale):
    """A scale of the logits of zero or next to it, over the smallest scale of a page: weights are alike."""
    pages = Pages(1, 2, 128, 320, 16, "e4m3", 1).fill([299], 2)
    pages.K_scale[pages.table[0, ::2].long()] = LEAST
    attend(ctx, pages, rows((1, n_q, 2, 128), dtype, 3), [299], dtype, scale)


@pytest.mark.parametrize("n_q", [1, 40, 70])
def test_zero_codes_with_the_largest_scale(ctx, n_q):
    """Large float32 queries over a page whose scale's product with them is past the largest float, but whose codes are zero."""
    pages = Pages(1, 2, 64, 160, 32, "i8", 1).fill([150], 2)
    at = pages.table[0].long()
    pages.K_scale[at] = 2.0 ** -27
    pages.K[at[1]], pages.K_scale[at[1]] = 0, 2.0 ** 122
    attend(ctx, pages, rows((1, n_q, 2, 64), "f32", 3) * 2.0 ** 20, [150], "f32", 1.0)
