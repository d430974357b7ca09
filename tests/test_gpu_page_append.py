"""Rows rotated, rounded to 8 bits and appended to pages, and read back out of them."""
import itertools
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_pages import DT, KIND, LEAST, MOST, ROTATION, SENTINEL, Pages, desc, i32, needed_exponent, rotary, rows, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def check_rows(pages, before, k, v, start, n, pos, r, code):
    """Every page after an append of rows k, v [B, T, H, d] against the rule; n[b] rows of sequence b to slots start[b] ..
    before: pages.state() of the start.  What the call does not touch, bit for bit."""
    B, H, d, N_cap = pages.shape
    want = [t.clone() for t in before]
    for b in range(B):
        if n[b] == 0:
            continue
        rot, size = (k[b, :n[b]].double(), 0) if r is None else turned(k[b, :n[b]], pos[b] + torch.arange(n[b], device="cuda"), r[0].dims,
                                                                       r[0].interleaved, r[1], r[2])
        slack = ROTATION * size if r is not None else torch.zeros_like(rot)
        for c in range(start[b] // pages.page, (start[b] + n[b] - 1) // pages.page + 1):
            at = int(pages.table[b, c])
            lo, hi = max(start[b], c * pages.page), min(start[b] + n[b], (c + 1) * pages.page)
            held, src = lo - c * pages.page, slice(lo - start[b], hi - start[b])
            for x, (codes, scales, new, err) in enumerate(((pages.K, pages.K_scale, rot, slack), (pages.V, pages.V_scale, v[b].double(), None))):
                new = new[src].transpose(0, 1)                                           # [H, rows, d]
                err = torch.zeros_like(new) if err is None else err[src].transpose(0, 1)
                old = before[2 + x][at].view(torch.float32)
                for h in range(H):
                    s = scales[at, h].item()
                    tops = [(new[h].abs() + side * err[h]).max().item() for side in (-1, 1)]
                    allowed = {2.0 ** needed_exponent(t, code) for t in tops}
                    if held:
                        allowed = {max(a, old[h].item()) for a in allowed}
                    assert s in allowed, (b, c, h, x, s, allowed)
                    got = codes[at, h, held:held + hi - lo].view(KIND[code]).double() * s
                    off = (got - new[h]).abs()
                    # half a step: of the scale, or of a value's own three bits, down to 2^-9 of the scale
                    half = s / 2 if code == "i8" else torch.clamp(2.0 ** -4 * (new[h].abs() + err[h]), min=2.0 ** -10 * s)
                    assert (off <= half + err[h]).all(), (b, c, h, x, (off / half).max().item())
                    if held and s > old[h].item():
                        was = before[x][at, h, :held].view(KIND[code]).float() * (old[h].item() / s)
                        again = was.round().to(torch.int8) if code == "i8" else was.to(torch.float8_e4m3fn)
                        want[x][at, h, :held] = again.view(torch.uint8)
                    want[x][at, h, held:held + hi - lo] = codes[at, h, held:held + hi - lo]
                    want[2 + x][at, h] = scales[at, h].view(torch.int32)
    for got, ref in zip(pages.state(), want):
        assert torch.equal(got, ref), "something that the call has no part in has changed"


def run_append(ctx, dtype, code, d, B, H, group, T, page, start, n_append=None, N_cap=None, dims=None, interleaved=False, seed=0, fused=False, gain=1.0,
               pos=None, spread=3):
    n = [T] * B if n_append is None else [min(max(x, 0), T) for x in n_append]
    N_cap = max(s + T for s in start) + 3 if N_cap is None else N_cap
    fits = [max(0, min(m, N_cap - s)) for m, s in zip(n, start)]
    pages = Pages(B, H, d, N_cap, page, code, seed).fill(start, seed + 1, spread)
    Hq = H * group
    x = rows((B, T, Hq + 2 * H, d), dtype, seed + 2) * gain
    q, k, v = (y.contiguous() for y in x.split([Hq, H, H], 2))
    q_out = torch.full_like(q, SENTINEL)
    r = None if dims is None else rotary(dims, interleaved)
    first = start if pos is None else pos
    before = pages.state()
    if fused:
        size = x.element_size() * d
        args = [x.data_ptr(), x.data_ptr() + Hq * size, x.data_ptr() + (Hq + H) * size, (Hq + 2 * H) * d]
    else:
        args = [q, k, v, 0]
    ctx.ig_append_pages(desc(B, H, d, max(start), N_cap, dtype), pages.struct(), r and r[0], group, T, *args, i32(n_append), i32(start), i32(pos), q_out)
    torch.cuda.synchronize()
    check_rows(pages, before, k, v, start, fits, first, r, code)
    for b in range(B):
        assert (q_out[b, n[b]:] == SENTINEL).all()
        if r is None:
            assert torch.equal(q_out[b, :n[b]], q[b, :n[b]])
        elif n[b]:
            ref, size = turned(q[b, :n[b]], first[b] + torch.arange(n[b], device="cuda"), dims, interleaved, r[1], r[2])
            tol = ROTATION * size + (2.0 ** -11 if dtype == "f16" else 2.0 ** -24) * ref.abs() + 2.0 ** -25
            assert ((q_out[b, :n[b]].double() - ref).abs() <= tol).all()
    return pages, k, v


@pytest.mark.parametrize("dtype,code", list(itertools.product(["f16", "f32"], ["i8", "e4m3"])))
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_prompts(ctx, dtype, code, d, page):
    """Into empty pages, and from the middle of one on."""
    run_append(ctx, dtype, code, d, B=3, H=3, group=2, T=151, page=page, start=[0, 5, 130], dims=d, seed=d + page)


@pytest.mark.parametrize("dtype,code", list(itertools.product(["f16", "f32"], ["i8", "e4m3"])))
@pytest.mark.parametrize("T", [1, 2, 7])
@pytest.mark.parametrize("dims,interleaved", [(None, False), (64, False), (64, True), (16, True), (24, False), (2, False)])
def test_few_rows(ctx, dtype, code, T, dims, interleaved):
    start = [0, 1, 15, 16, 31, 500]
    run_append(ctx, dtype, code, 64, B=6, H=9, group=1, T=T, page=16, start=start, dims=dims, interleaved=interleaved, seed=T, gain=3.0)


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dims,interleaved", [(128, False), (128, True), (40, False), (20, False), (6, False), (20, True), (None, False)])
def test_ragged(ctx, fused, dims, interleaved):
    """Counts of zero and out of range, sequences that end at their capacity or behind it, positions of the caller's."""
    run_append(ctx, "f16", "i8", 128, B=6, H=2, group=4, T=40, page=32, start=[0, 90, 70, 100, 99, 33], n_append=[40, 40, 0, 5, -3, 1000], N_cap=100,
               dims=dims, interleaved=interleaved, fused=fused, pos=[7, 0, 1 << 17, 5, 5, 100])


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("gain", [2.0 ** -20, 2.0 ** 10, 1e30, 0.0])
def test_sizes_of_values(ctx, code, gain):
    """Scales grow by many powers of two at once, or not at all."""
    run_append(ctx, "f32", code, 64, B=2, H=2, group=1, T=5, page=16, start=[3, 30], dims=64, gain=gain)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_borders_of_the_scale(ctx, code):
    """A largest value of exactly 127 (448) codes, and the next float above it."""
    for top, e in ((MOST[code], 0), (MOST[code] * 2.0 ** -7, -7), (math.nextafter(MOST[code], 1e9), None), (2.0 ** -126, -80), (MOST[code] * LEAST, -80)):
        pages = Pages(1, 1, 32, 16, 16, code, 1)
        k = torch.zeros((1, 1, 1, 32), device="cuda")
        k[..., 3] = -top
        up = torch.tensor(top).nextafter(torch.tensor(math.inf)).item() if e is None else top
        k[..., 3] = -up
        ctx.ig_append_pages(desc(1, 1, 32, 0, 16, "f32"), pages.struct(), None, 1, 1, None, k, k, 0, None, None, None, None)
        torch.cuda.synchronize()
        at = int(pages.table[0, 0])
        assert pages.K_scale[at, 0].item() == 2.0 ** (1 if e is None else e) == pages.V_scale[at, 0].item()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_not_finite(ctx, dtype, code):
    """NaN and infinities are stored as 0 and do not count for the scale."""
    T, d = 20, 64
    clean = rows((1, T, 2, d), dtype, 1)
    bad = clean.clone()
    bad[0, 3, 0, 5], bad[0, 4, 1, 6], bad[0, 19, 0, 0] = math.nan, math.inf, -math.inf
    clean[0, 3, 0, 5], clean[0, 4, 1, 6], clean[0, 19, 0, 0] = 0, 0, 0
    states = []
    for k in (clean, bad):
        pages = Pages(1, 2, d, 32, 16, code, 1)
        ctx.ig_append_pages(desc(1, 2, d, 0, 32, dtype), pages.struct(), None, 1, T, None, k, k, 0, None, None, None, None)
        torch.cuda.synchronize()
        states.append(pages.state())
    for a, b in zip(*states):
        assert torch.equal(a, b)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_token_by_token(ctx, code, dtype):
    """Values of rising size one by one: every row stays within one scale (e4m3: 2^-4 of itself and 2^-9 of a scale), and the
    scales are those of one call for all of them."""
    B, H, d, T, page = 2, 3, 64, 32, 32
    k = rows((B, T, H, d), dtype, 1) * (1.2 ** torch.arange(T, device="cuda")).to(DT[dtype])[:, None, None]
    v = rows((B, T, H, d), dtype, 2) * (1.3 ** torch.arange(T, device="cuda")).to(DT[dtype])[:, None, None]
    one, all_at_once = Pages(B, H, d, T, page, code, 1), Pages(B, H, d, T, page, code, 1)
    for t in range(T):
        ctx.ig_append_pages(desc(B, H, d, t, T, dtype), one.struct(), None, 1, 1, None, k[:, t:t + 1].contiguous(), v[:, t:t + 1].contiguous(), 0,
                            None, None, None, None)
    ctx.ig_append_pages(desc(B, H, d, 0, T, dtype), all_at_once.struct(), None, 1, T, None, k, v, 0, None, None, None, None)
    torch.cuda.synchronize()
    mine = one.table.view(-1).long()
    for x, rows_ in (("K", k), ("V", v)):
        assert torch.equal(getattr(one, x + "_scale")[mine], getattr(all_at_once, x + "_scale")[mine])
        for b in range(B):
            ref = rows_[b].double().transpose(0, 1)
            s = getattr(one, x + "_scale")[one.table[b, 0].long()].double()[:, None, None]
            err = (one.values(x, b, T) - ref).abs()
            bound = s * torch.ones_like(err) if code == "i8" else 2.0 ** -4 * ref.abs() + 2.0 ** -9 * s
            assert (err < bound).all(), (err / bound).max()


def test_entries_outside_the_pool(ctx):
    """Nothing is written through them; the other pages get their rows."""
    B, H, d, T, page = 2, 2, 64, 48, 16
    k = rows((B, T, H, d), "f16", 1)
    good, bad = Pages(B, H, d, T, page, "i8", 1), Pages(B, H, d, T, page, "i8", 1)
    skipped = [int(bad.table[0, 1]), int(bad.table[1, 2])]
    bad.table[0, 1], bad.table[1, 2] = -1, bad.K.shape[0]
    for p in (good, bad):
        ctx.ig_append_pages(desc(B, H, d, 0, T, "f16"), p.struct(), None, 1, T, None, k, k, 0, None, None, None, None)
    torch.cuda.synchronize()
    untouched = Pages(B, H, d, T, page, "i8", 1).state()
    for a, b, u in zip(good.state(), bad.state(), untouched):
        a[skipped] = u[skipped]
        assert torch.equal(a, b)


@pytest.mark.parametrize("dims,interleaved", [(64, False), (24, False), (64, True)])
def test_queries_in_place(ctx, dims, interleaved):
    B, H, d, T = 2, 2, 64, 9
    q, k = rows((B, T, 3 * H, d), "f16", 1), rows((B, T, H, d), "f16", 2)
    r, out, lens = rotary(dims, interleaved), torch.zeros_like(q), i32([9, 4])
    apart = q.clone()
    for to, src in ((out, apart), (q, q)):
        pages = Pages(B, H, d, 16, 16, "i8", 1)
        if to is out:
            to.copy_(q)
        ctx.ig_append_pages(desc(B, H, d, 0, 16, "f16"), pages.struct(), r[0], 3, T, src, k, k, 0, lens, None, i32([5, 6]), to)
    torch.cuda.synchronize()
    assert torch.equal(out, q)


@pytest.mark.parametrize("dtype,code", list(itertools.product(["f16", "f32"], ["i8", "e4m3"])))
@pytest.mark.parametrize("d,page", [(32, 16), (64, 128), (128, 32), (256, 64)])
def test_rows_read_back(ctx, dtype, code, d, page):
    """Lists with counts of zero and past the stride, slots out of range, the same slot twice."""
    B, H, N_cap, stride = 3, 4, 300, 77
    pages = Pages(B, H, d, N_cap, page, code, 1).fill([N_cap] * B, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    idx = torch.randint(0, N_cap, (B * H, stride), generator=g, device="cuda").int()
    idx[:, 3], idx[:, 4], idx[:, 5], idx[:, 6] = -9, 1 << 30, 17, 17
    cnt = torch.randint(0, stride + 1, (B * H,), generator=g, device="cuda").int()
    cnt[0], cnt[1], cnt[2] = 0, stride, stride + 50
    K, V = (torch.full((B * H, stride, d), SENTINEL, dtype=DT[dtype], device="cuda") for _ in "KV")
    ctx.ig_gather_pages(desc(B, H, d, N_cap, N_cap, dtype), pages.struct(), idx, stride, cnt, K, V)
    torch.cuda.synchronize()
    for x, got in (("K", K), ("V", V)):
        for b in range(B):
            values = pages.values(x, b, N_cap)
            for h in range(H):
                i, n = b * H + h, min(int(cnt[b * H + h]), stride)
                assert torch.equal(got[i, :n], values[h, idx[i, :n].clamp(0, N_cap - 1).long()].to(DT[dtype]))
                assert (got[i, n:] == SENTINEL).all()


def test_entries_outside_the_pool_are_clamped_for_reading(ctx):
    B, H, d, N = 1, 1, 64, 64
    pages = Pages(B, H, d, N, 16, "i8", 1).fill([N], 2)
    pages.K_scale.nan_to_num_(1.0), pages.V_scale.nan_to_num_(1.0)
    idx, cnt = i32([list(range(N))]), i32([N])
    ds = desc(B, H, d, N, N, "f32")
    for entry, means in ((-3, 0), (99, pages.K.shape[0] - 1)):
        results = []
        for e in (entry, means):
            pages.table[0, 2] = e
            K, V = (torch.zeros((1, N, d), device="cuda") for _ in "KV")
            ctx.ig_gather_pages(ds, pages.struct(), idx, N, cnt, K, V)
            torch.cuda.synchronize()
            results.append((K, V))
        assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
