"""Attention over pages of 8-bit codes against the definition in 64 bits."""
import itertools

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import SENTINEL, desc, i32, rows
from ig_pages import Pages, check_attention, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_one_token(ctx, dtype, code, d, page):
    run_attention(ctx, dtype, code, d, B=2, H=3, group=1, n_q=1, N=333, N_cap=340, page=page, seed=d + page)


@pytest.mark.parametrize("code,dtype", list(itertools.product(["i8", "e4m3"], ["f16", "f32"])))
@pytest.mark.parametrize("d,group,n_q", [(128, 4, 1), (64, 8, 2), (128, 5, 5), (32, 1, 31), (256, 2, 9), (128, 1, 33), (64, 4, 40),
                                         (256, 3, 45), (128, 2, 150), (32, 2, 200)])
def test_row_blocks(ctx, code, dtype, d, group, n_q):
    """From a few query rows to more than a workgroup's, grouped heads, an odd number of slots."""
    run_attention(ctx, dtype, code, d, B=2, H=2, group=group, n_q=n_q, N=291, N_cap=291, page=32, seed=n_q)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n_q", [1, 7, 70])
@pytest.mark.parametrize("page", [16, 64])
def test_ragged(ctx, dtype, n_q, page):
    """Lengths of zero, one and past N; query lengths of zero and past n_q; queries before the first slot see nothing."""
    N = 200
    kv, nq = [0, 1, 17, 200, 64, 63, 3], [n_q, 1, n_q, n_q, 0, max(1, n_q - 3), n_q]
    run_attention(ctx, dtype, "e4m3", 64, B=7, H=2, group=2, n_q=n_q, N=N, N_cap=208, page=page, kv=kv, nq=nq, seed=5)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("B,H,group,n_q,N", [(1, 2, 1, 1, 5000), (3, 1, 4, 1, 9000), (1, 1, 8, 3, 20000), (2, 1, 4, 100, 3000), (1, 1, 1, 1, 1)])
def test_slices(ctx, dtype, B, H, group, n_q, N):
    kv = [max(1, N - b * (N // 3)) for b in range(B)] if B > 1 else None
    for code in ("i8", "e4m3"):
        run_attention(ctx, dtype, code, 128, B, H, group, n_q, N, N + 3, 64, kv=kv, seed=N)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n_q", [1, 40])
def test_scales_far_apart(ctx, dtype, n_q):
    """Pages whose scales differ by 2^40: what counts is a weight times its scale."""
    for code in ("i8", "e4m3"):
        B, H, d, N = 1, 2, 64, 300
        pages = Pages(B, H, d, N, 32, code, 3).fill([N], 4)
        pages.V_scale[pages.table[0, 1::3].long()] *= 2.0 ** -40
        pages.V_scale[pages.table[0, 2::3].long()] *= 2.0 ** -20
        q = rows((B, n_q, H, d), dtype, 5)
        out = torch.full_like(q, SENTINEL)
        ctx.ig_page_attention(desc(B, H, d, N, N, dtype, 0.125), pages.struct(), 1, n_q, q, None, None, out)
        torch.cuda.synchronize()
        check_attention(pages, q, [N], [n_q], 1, 0.125, dtype, out, out)
        # and a row that sees small ones alone
        only = torch.full_like(q[:, :1], SENTINEL)
        pages.V_scale[pages.table[0, 0].long()] *= 2.0 ** -60
        ctx.ig_page_attention(desc(B, H, d, 32, 32, dtype, 0.125), pages.struct(), 1, 1, q[:, :1].contiguous(), None, None, only)
        torch.cuda.synchronize()
        if dtype == "f32":
            check_attention(pages, q[:, :1], [32], [1], 1, 0.125, dtype, only, only)


@pytest.mark.parametrize("scale", [-0.5, 0.0, 3.0])
@pytest.mark.parametrize("n_q", [1, 50])
def test_signs_of_the_scale(ctx, scale, n_q):
    for dtype in ("f16", "f32"):
        run_attention(ctx, dtype, "i8", 64, 1, 2, 2, n_q, 100, 100, 16, scale=scale, spread=1)


@pytest.mark.parametrize("n_q", [1, 48])
def test_entries_outside_the_pool(ctx, n_q):
    """Table entries past a sequence's pages are not looked at; among them they are read as the nearest page."""
    B, H, d, N, page = 2, 2, 64, 100, 16
    pages = Pages(B, H, d, 160, page, "i8", 1).fill([N, N], 2)
    q = rows((B, n_q, H, d), "f16", 3)
    out, other = torch.full_like(q, SENTINEL), torch.full_like(q, SENTINEL)
    ds = desc(B, H, d, N, 160, "f16", 0.125)
    ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, out)
    pages.table[:, 7:] = 1 << 30
    ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, other)
    torch.cuda.synchronize()
    assert torch.equal(out, other)
    for entry, means in ((-5, 0), (1 << 30, pages.K.shape[0] - 1)):
        pages.table[1, 2] = entry
        ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, out)
        pages.table[1, 2] = means
        pages.K_scale.nan_to_num_(1.0), pages.V_scale.nan_to_num_(1.0)
        ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, other)
        torch.cuda.synchronize()
        assert torch.equal(out[0], other[0])
        ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, out)
        torch.cuda.synchronize()
        assert torch.equal(out, other)


def test_odd_scales_are_read_as_powers_of_two(ctx):
    B, H, d, N = 1, 2, 64, 64
    pages = Pages(B, H, d, N, 32, "i8", 1).fill([N], 2)
    q = rows((B, 1, H, d), "f16", 3)
    out, other = torch.zeros_like(q), torch.zeros_like(q)
    ds = desc(B, H, d, N, N, "f16", 0.125)
    ctx.ig_page_attention(ds, pages.struct(), 1, 1, q, None, None, out)
    pages.K_scale *= 1.9
    pages.V_scale *= 1.2
    ctx.ig_page_attention(ds, pages.struct(), 1, 1, q, None, None, other)
    torch.cuda.synchronize()
    assert torch.equal(out, other)


@pytest.mark.parametrize("n_q", [1, 60])
def test_repeatable_and_on_another_stream(ctx, n_q):
    a = run_attention(ctx, "f16", "i8", 128, 3, 2, 2, n_q, 2000, 2000, 32, kv=[2000, 400, 1])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    b = run_attention(ctx, "f16", "i8", 128, 3, 2, 2, n_q, 2000, 2000, 32, kv=[2000, 400, 1], stream=s)
    assert torch.equal(a, b)


def test_no_slots(ctx):
    """N = 0: every query sees nothing."""
    pages = Pages(2, 2, 64, 16, 16, "e4m3", 1)
    for n_q in (1, 50):
        q = rows((2, n_q, 2, 64), "f16", 3)
        out = torch.full_like(q, SENTINEL)
        ctx.ig_page_attention(desc(2, 2, 64, 0, 16, "f16"), pages.struct(), 1, n_q, q, i32([n_q, 0]), None, out)
        torch.cuda.synchronize()
        assert (out[0] == 0).all() and (out[1] == SENTINEL).all()


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("d,n_q,N", [(32, 150, 160), (64, 290, 300), (64, 300, 400), (128, 150, 160)])
def test_many_workgroups(ctx, code, d, n_q, N):
    """Prompts of many heads: row blocks in pairs, two row blocks a wave; the last rows see all, the first none or few."""
    kv = [N, N, 1, N - 70, n_q - 9, N, 64, N]
    run_attention(ctx, "f16", code, d, B=8, H=64, group=1, n_q=n_q, N=N, N_cap=N, page=16, kv=kv, seed=d)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_rows(ctx, d):
    """A chunk over many tiles: references that rise again and again, rows with one large logit."""
    B, H, n_q, N = 1, 2, 200, 5000
    pages = Pages(B, H, d, N, 64, "i8", 1).fill([N], 2, spread=1)
    # keys grow along the sequence, so that every tile raises the largest logit
    for c in range(-(-N // 64)):
        pages.K_scale[int(pages.table[0, c])] = 2.0 ** (-9 + c // 16)
    q = rows((B, n_q, H, d), "f16", 3)
    out = torch.full_like(q, SENTINEL)
    ctx.ig_page_attention(desc(B, H, d, N, N, "f16", 0.5), pages.struct(), 1, n_q, q, None, None, out)
    torch.cuda.synchronize()
    check_attention(pages, q, [N], [n_q], 1, 0.5, "f16", out, out)


@pytest.mark.parametrize("n_q", [1, 40])
def test_what_lies_behind_the_last_slot(ctx, n_q):
    """Junk codes (e4m3: NaN) and scales behind a sequence's slots, in its last page and in entries past it, do not count."""
    B, H, d, N, page = 2, 2, 64, 70, 32
    for dtype in ("f16", "f32"):
        pages = Pages(B, H, d, 128, page, "e4m3", 1).fill([N, 33], 2)
        q = rows((B, n_q, H, d), dtype, 3)
        out, other = torch.full_like(q, SENTINEL), torch.full_like(q, SENTINEL)
        ds = desc(B, H, d, N, 128, dtype, 0.125)
        ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, i32([N, 33]), out)
        for b, n in enumerate((N, 33)):
            at = int(pages.table[b, n // page])
            pages.K[at, :, n % page:], pages.V[at, :, n % page:] = 0x11, 0x22
            rest = pages.table[b, n // page + 1:].long()
            pages.K[rest], pages.V[rest], pages.K_scale[rest], pages.V_scale[rest] = 0x33, 0x44, 1.0, 1.0
        ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, i32([N, 33]), other)
        torch.cuda.synchronize()
        assert torch.isfinite(out).all() and torch.equal(out, other)


def test_shared_pages(ctx):
    """Two sequences with the same first pages, and the same page twice in one."""
    B, H, d, page, N = 2, 2, 128, 16, 64
    pages = Pages(B, H, d, N, page, "i8", 1).fill([N, N], 2)
    pages.table[1, :2] = pages.table[0, :2]
    pages.table[0, 3] = pages.table[0, 2]
    for n_q in (1, 50):
        q = rows((B, n_q, H, d), "f16", 3)
        out = torch.full_like(q, SENTINEL)
        ctx.ig_page_attention(desc(B, H, d, N, N, "f16", 0.1), pages.struct(), 1, n_q, q, None, None, out)
        torch.cuda.synchronize()
        check_attention(pages, q, [N, N], [n_q, n_q], 1, float(torch.tensor(0.1)), "f16", out, out)


def test_pages_far_into_the_pool(ctx):
    """Codes past 2^32 bytes, and scales past 2^16 pages."""
    H, d, page, n = 8, 128, 128, 40000                         # 5.2 GB of K
    K = torch.zeros((n, H, page, d), dtype=torch.uint8, device="cuda")
    V = torch.zeros_like(K)
    scales = [torch.ones((n, H), device="cuda") for _ in "KV"]
    small = Pages(1, H, d, 256, page, "i8", 1).fill([256], 2)
    far = [n - 1, 33333]
    for x, y, s, t in ((K, small.K, scales[0], small.K_scale), (V, small.V, scales[1], small.V_scale)):
        for c, at in enumerate(far):
            x[at], s[at] = y[int(small.table[0, c])], t[int(small.table[0, c])]
    table = i32([far])
    for n_q in (1, 40):
        q = rows((1, n_q, H, d), "f16", 3)
        out, other = torch.zeros_like(q), torch.zeros_like(q)
        ds = desc(1, H, d, 256, 256, "f16", 0.1)
        ctx.ig_page_attention(ds, small.struct(), 1, n_q, q, None, None, out)
        ctx.ig_page_attention(ds, ig.IgPages(table, K, V, *scales, ig.IG_CODE_I8), 1, n_q, q, None, None, other)
        torch.cuda.synchronize()
        assert torch.equal(out, other)
    # appended to and read back there
    k = rows((1, 3, H, d), "f16", 5)
    idx, cnt = i32([[200, 201, 202]] * H), i32([3] * H)
    got = []
    for p in (small.struct(), ig.IgPages(table, K, V, *scales, ig.IG_CODE_I8)):
        to = [torch.zeros((H, 3, d), dtype=torch.float16, device="cuda") for _ in "KV"]
        ctx.ig_append_pages(desc(1, H, d, 200, 256, "f16"), p, None, 1, 3, None, k, k, 0, None, None, None, None)
        ctx.ig_gather_pages(desc(1, H, d, 256, 256, "f16"), p, idx, 3, cnt, *to)
        torch.cuda.synchronize()
        got.append(to)
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and got[0][0].any()


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_float32_rows_in_blocks_of_32(ctx, code, d):
    """Enough turns to fill the GPU with: two blocks of 16 rows a wave, in slices too."""
    run_attention(ctx, "f32", code, d, B=4, H=4, group=2, n_q=41, N=3000, N_cap=3000, page=32, kv=[3000, 1500, 41, 7], nq=[41, 33, 41, 9], seed=d)
    run_attention(ctx, "f32", code, d, B=8, H=16, group=1, n_q=130, N=130, N_cap=140, page=16, seed=d + 1)


def test_half_precision_rows_in_several_blocks(ctx):
    """33 to 64 rows, and 17 to 64 at d = 256: row blocks over the same codes."""
    for code, d, n_q in (("i8", 128, 17), ("e4m3", 64, 32), ("i8", 256, 9), ("e4m3", 256, 31), ("i8", 32, 20)):
        run_attention(ctx, "f16", code, d, B=3, H=2, group=2, n_q=n_q, N=1000, N_cap=1000, page=128, kv=[1000, 300, 5], seed=n_q)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n_q", [1, 70])
def test_scales_at_the_ends_of_their_range(ctx, dtype, n_q):
    """Pages of zero codes with the largest scales, and of the smallest, beside ordinary ones."""
    B, H, d, N = 1, 2, 64, 160
    pages = Pages(B, H, d, N, 32, "i8", 3).fill([N], 4)
    at = pages.table[0].long()
    pages.K[at[1]], pages.V[at[1]], pages.K_scale[at[1]], pages.V_scale[at[1]] = 0, 0, 2.0 ** 122, 2.0 ** 122
    pages.K_scale[at[2]], pages.V_scale[at[2]] = 2.0 ** -80, 2.0 ** -80
    q = rows((B, n_q, H, d), dtype, 5)
    out, plain = torch.full_like(q, SENTINEL), torch.full_like(q, SENTINEL)
    ds = desc(B, H, d, N, N, dtype, 8.0)
    ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, out)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    # keys of zero codes have logits of zero whatever their scale; their values are zero, so they only take weight
    pages.K_scale[at[1]] = 1.0
    ctx.ig_page_attention(ds, pages.struct(), 1, n_q, q, None, None, plain)
    torch.cuda.synchronize()
    assert torch.equal(out, plain)
