"""Rotary embedding of rows on the device against the definition in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_pages import DT, ROTATION, SENTINEL, i32, rotary, rows, turned

pytestmark = pytest.mark.gpu
TYPE = {"f16": ig.IG_F16, "f32": ig.IG_F32}


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def check(got, x, pos, r, dtype, inverse=False):
    """Rotated channels to the rounding of the rotation and their own; the others bit for bit."""
    st, freq, magnitude = r
    ref, size = turned(x, pos, st.dims, st.interleaved, freq, magnitude, inverse)
    tol = ROTATION * size + (2.0 ** -11 if dtype == "f16" else 2.0 ** -24) * ref.abs() + (2.0 ** -25 if dtype == "f16" else 2.0 ** -126)
    err = (got.double() - ref).abs()
    assert (err <= tol).all(), f"off by {(err / tol).max().item():.2f} tolerances"
    assert torch.equal(got[..., st.dims:], x[..., st.dims:])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("inverse", [0, 1])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,dims", [(16, 2), (16, 16), (32, 8), (64, 64), (64, 32), (80, 20), (96, 48), (128, 128), (128, 40), (256, 64), (1024, 1024)])
def test_layouts(ctx, dtype, inverse, interleaved, d, dims):
    n, heads = 37, 11
    x = rows((n, heads, d), dtype, d + dims)
    pos = torch.randint(-5, 1 << 20, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).int()
    r = rotary(dims, interleaved)
    out = torch.full_like(x, SENTINEL)
    ctx.ig_rotate_rows(TYPE[dtype], n, heads, d, r[0], inverse, pos, x, 0, out, 0)
    torch.cuda.synchronize()
    check(out, x, pos, r, dtype, inverse)
    # in place
    y = x.clone()
    ctx.ig_rotate_rows(TYPE[dtype], n, heads, d, r[0], inverse, pos, y, 0, y, 0)
    torch.cuda.synchronize()
    assert torch.equal(y, out)


@pytest.mark.parametrize("pos", [[0], [1], [2 ** 31 - 1], [-2 ** 31], [131071]])
@pytest.mark.parametrize("heads", [1, 8, 9])
def test_one_token(ctx, pos, heads):
    x = rows((1, heads, 64), "f32", 3)
    r, out = rotary(64), torch.zeros_like(x)
    ctx.ig_rotate_rows(ig.IG_F32, 1, heads, 64, r[0], 0, i32(pos), x, 0, out, 0)
    torch.cuda.synchronize()
    st, freq, magnitude = r
    ref, size = turned(x, i32(pos), 64, False, freq, magnitude)
    # (the angle itself, at most 2^31, is a double: half a step of 2^-22)
    assert ((out.double() - ref).abs() <= (ROTATION + 2.0 ** -22) * size).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("interleaved,dims", [(False, 64), (True, 64), (False, 24)])
def test_strides(ctx, dtype, interleaved, dims):
    """Rows in the middle of a wider buffer, into another one, and in place; what lies around them stays."""
    n, heads, d, wide, wider = 13, 3, 64, 5 * 64, 7 * 64
    x, to = rows((n, wide), dtype, 1), torch.full((n, wider), SENTINEL, dtype=DT[dtype], device="cuda")
    pos, r = i32(list(range(100, 100 + n))), rotary(dims, interleaved)
    mine = x[:, 64:64 + heads * d].reshape(n, heads, d)
    size = x.element_size()
    ctx.ig_rotate_rows(TYPE[dtype], n, heads, d, r[0], 0, pos, x.data_ptr() + 64 * size, wide, to.data_ptr() + 128 * size, wider)
    torch.cuda.synchronize()
    check(to[:, 128:128 + heads * d].reshape(n, heads, d), mine, pos, r, dtype)
    assert (to[:, :128] == SENTINEL).all() and (to[:, 128 + heads * d:] == SENTINEL).all()
    y = x.clone()
    ctx.ig_rotate_rows(TYPE[dtype], n, heads, d, r[0], 0, pos, y.data_ptr() + 64 * size, wide, y.data_ptr() + 64 * size, wide)
    torch.cuda.synchronize()
    assert torch.equal(y[:, 64:64 + heads * d], to[:, 128:128 + heads * d]) and torch.equal(y[:, :64], x[:, :64])
    assert torch.equal(y[:, 64 + heads * d:], x[:, 64 + heads * d:])


@pytest.mark.parametrize("kind,more", [(ig.IG_ROPE_LINEAR, dict(factor=4.0)), (ig.IG_ROPE_NTK, dict(factor=4.0)),
                                       (ig.IG_ROPE_RAMP, dict(factor=8.0, low=1.0, high=32.0, original=2048)),
                                       (ig.IG_ROPE_WAVELENGTH, dict(factor=8.0, low=1.0, high=4.0, original=2048))])
def test_stretched(ctx, kind, more):
    n, heads, d = 50, 4, 128
    x, r = rows((n, heads, d), "f32", 1), rotary(d, kind=kind, **more)
    pos, out = i32([k * 1311 for k in range(n)]), torch.zeros_like(x)
    ctx.ig_rotate_rows(ig.IG_F32, n, heads, d, r[0], 0, pos, x, 0, out, 0)
    torch.cuda.synchronize()
    check(out, x, pos, r, "f32")


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(ctx, interleaved):
    """inverse = 1 is the transpose: against the formula's and against differences."""
    n, heads, d, dims = 6, 2, 32, 16
    r = rotary(dims, interleaved, ig.IG_ROPE_RAMP, factor=4.0, low=1.0, high=8.0, original=64)
    assert r[2] > 1
    x, dy, pos = rows((n, heads, d), "f32", 1), rows((n, heads, d), "f32", 2), i32([0, 5, 77, 78, 1000, 50000])
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    ctx.ig_rotate_rows(ig.IG_F32, n, heads, d, r[0], 1, pos, dy, 0, dx, 0)
    torch.cuda.synchronize()
    leaf = x.double().requires_grad_()
    a = slice(0, dims, 2) if interleaved else slice(0, dims // 2)
    b = slice(1, dims, 2) if interleaved else slice(dims // 2, dims)
    angle = pos.double()[:, None, None] * torch.from_numpy(r[1]).cuda()
    cos, sin = angle.cos() * r[2], angle.sin() * r[2]
    loss = ((leaf[..., a] * cos - leaf[..., b] * sin) * dy[..., a]).sum() + ((leaf[..., b] * cos + leaf[..., a] * sin) * dy[..., b]).sum() + \
        (leaf[..., dims:] * dy[..., dims:]).sum()
    loss.backward()
    size = turned(dy, pos, dims, interleaved, r[1], r[2])[1] + dy.double().abs()
    assert ((dx.double() - leaf.grad).abs() <= (ROTATION + 2.0 ** -24) * size).all()
    # The operator is linear: a step of 1/8 in one value changes the sum of dy y by 1/8 of its gradient, to both passes' rounding.
    step, at = 0.125, (2, 1, 3)
    sums = []
    for sign in (1, -1):
        moved = x.clone()
        moved[at] += sign * step
        ctx.ig_rotate_rows(ig.IG_F32, n, heads, d, r[0], 0, pos, moved, 0, y, 0)
        torch.cuda.synchronize()
        sums.append((y.double() * dy.double())[at[0], at[1]].sum().item())
    size = turned(x, pos, dims, interleaved, r[1], r[2])[1][at[0], at[1]] + x.double().abs()[at[0], at[1]] + step * r[2]
    slack = 2 * ((ROTATION + 2.0 ** -24) * size * dy.double().abs()[at[0], at[1]]).sum().item() / (2 * step)
    assert abs((sums[0] - sums[1]) / (2 * step) - dx[at].item()) <= slack + 2.0 ** -20


def test_values_that_stay(ctx):
    """Infinities and NaN past the rotated channels stay where they are."""
    x = rows((3, 2, 64), "f16", 1)
    x[..., 24], x[..., 40], x[..., 63] = math.inf, math.nan, -math.inf
    for interleaved in (False, True):
        r, out = rotary(24, interleaved), torch.zeros_like(x)
        ctx.ig_rotate_rows(ig.IG_F16, 3, 2, 64, r[0], 0, i32([1, 2, 3]), x, 0, out, 0)
        torch.cuda.synchronize()
        assert torch.isfinite(out[..., :24]).all() and torch.equal(out[..., 24:].nan_to_num(9.0, 8.0, 7.0), x[..., 24:].nan_to_num(9.0, 8.0, 7.0))


def test_like_the_rehearsals_host_call(ctx):
    """The same rotation as ig_rope_rows, which a rotary model's queries are prepared with."""
    n, H, d = 9, 3, 128
    q = np.random.default_rng(1).standard_normal((n, H, d)).astype(np.float32)
    pos = np.arange(n, dtype=np.int32) * 1000
    want = ig.ig_rope_rows(q, pos)
    x, out = torch.from_numpy(q).cuda(), torch.zeros((n, H, d), device="cuda")
    ctx.ig_rotate_rows(ig.IG_F32, n, H, d, rotary(d)[0], 0, torch.from_numpy(pos).cuda(), x, 0, out, 0)
    size = turned(x, torch.from_numpy(pos).cuda(), d, False, rotary(d)[1], 1.0)[1]
    assert ((out.double() - torch.from_numpy(want).cuda().double()).abs() <= (ROTATION + 2.0 ** -24) * size).all()
