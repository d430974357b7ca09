"""Weights far below a row's largest that matter together, logits far out, and values that do not average out."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import DT, definition, desc, rows, weight_error

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def call(ctx, dtype, d, n_q, N, q, K, V, scale, tree):
    """One pool; tree: n_q nodes that see the pool and each other's first node, which holds nothing new."""
    out = torch.zeros_like(q)
    if tree:
        kt, vt = K[:, :, :1].expand(1, 1, n_q, d).transpose(1, 2).contiguous(), V[:, :, :1].expand(1, 1, n_q, d).transpose(1, 2).contiguous()
        bits = torch.ones((1, n_q), dtype=torch.int64, device="cuda")
        ctx.ig_tree_attention(desc(1, 1, d, N, N, dtype, scale), 1, n_q, q, kt, vt, bits, None, K, V, None, out)
    else:
        ctx.ig_cache_attention(desc(1, 1, d, N, N, dtype, scale), 1, n_q, q, None, K, V, None, None, out)
    torch.cuda.synchronize()
    return out


# (n_q, N, tree): attend_stream, attend_prompt with four and with eight waves
FORMS = [(1, 2048, False), (9, 2048, False), (30, 2048, False), (40, 2048, False), (200, 2048, False), (12, 2048, True), (60, 2048, True)]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("form", FORMS, ids=[f"{'tree' if f[2] else 'rows'}{f[0]}" for f in FORMS])
def test_small_weights_count(ctx, dtype, d, form):
    """In every run of 32 slots one with a value of zero outweighs the others by about 2^24, and the others' values
    alone, all of one sign, make the output."""
    n_q, N, tree = form
    g = torch.Generator(device="cuda").manual_seed(d)
    K = torch.zeros((1, 1, N, d), device="cuda")
    K[..., 0] = -24.0 - torch.rand((1, 1, N), generator=g, device="cuda")
    V = 900 + 100 * torch.rand((1, 1, N, d), generator=g, device="cuda")
    K[:, :, ::32], V[:, :, ::32] = 0, 0
    q = torch.zeros((1, n_q, 1, d), device="cuda")
    q[..., 0] = 1
    q, K, V = (x.to(DT[dtype]) for x in (q, K, V))
    scale = math.log(2.0)
    out = call(ctx, dtype, d, n_q, N, q, K, V, scale, tree)
    Kt, Vt = (torch.cat([x[0, 0], x[0, 0, :1]]) if tree else x[0, 0] for x in (K, V))
    i = torch.arange(n_q, device="cuda")
    sees = torch.ones((n_q, N + 1), dtype=torch.bool, device="cuda") if tree else torch.arange(N, device="cuda") <= (N - n_q + i)[:, None]
    ref, p, absum, size = definition(q[0, :, 0], Kt, Vt, sees, float(torch.tensor(scale, dtype=torch.float32)))
    n = Kt.shape[0]
    # as in ig_cache: the output's rounding, the weights' error and the sum's; and in half precision the weights' rounding,
    # half a step of 2^-10, or 2^-34 of the largest weight for those below 2^-23 of it
    e = weight_error(size, n, d) + n * 2.0 ** -24
    if dtype == "f16":
        tol = 2.0 ** -11 * ref.abs() + (e + 2.0 ** -11) * absum + n * 2.0 ** -34 * p.amax(1, keepdim=True) * Vt.double().abs().max() + 2.0 ** -25
    else:
        tol = 2.0 ** -24 * ref.abs() + e * absum + 2.0 ** -126
    assert (tol < 0.05 * ref).all()                # (what vanishes, or is a quarter off, is seen)
    err = (out[0, :, 0].double() - ref).abs()
    assert (err <= tol).all(), f"{(err / tol).max().item():.2f} tolerances"


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", [2.0 ** 17, 2.0 ** 19, 2.0 ** 20, 2.0 ** 21, 2.0 ** 23, 2.0 ** 25, 1e8])
@pytest.mark.parametrize("n_q,N", [(1, 300), (40, 300), (200, 700)])
def test_logits_far_out(ctx, dtype, sign, size, n_q, N):
    """Every seventh slot has a logit of `size` and the same values, the others have 3/8 to 6/8 of it: those values come
    out whole."""
    d = 64
    g = torch.Generator(device="cuda").manual_seed(1)
    K = torch.zeros((1, 1, N, d), device="cuda")
    K[..., 0] = 3 + torch.randint(0, 4, (1, 1, N), generator=g, device="cuda")       # logits 3/8 .. 6/8 of size ..
    K[..., 0][:, :, ::7] = 8                                                          # .. and some of size
    K *= sign
    V = rows((1, 1, N, d), "f32", 2)
    V[:, :, ::7] = V[:, :, :1].clone()
    q = torch.zeros((1, n_q, 1, d), device="cuda")
    q[..., 0] = 8
    q, K, V = (x.to(DT[dtype]) for x in (q, K, V))
    out = call(ctx, dtype, d, n_q, N, q, K, V, sign * size / 64, False)
    # the others' weights are 2^-(size / 4) at most and equal weights' sums are off by N half steps
    want = V[0, 0, 0].double()
    tol = (2.0 ** -11 if dtype == "f16" else 2.0 ** -24) * want.abs() + (2 * N + 8) * 2.0 ** -24 * want.abs()
    if dtype == "f16":
        tol = tol + 2.0 ** -11 * want.abs() + 2.0 ** -25
    assert ((out[0, :, 0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n_q,N", [(1, 100000), (70, 60000)])
def test_long_with_values_of_one_sign(ctx, dtype, n_q, N):
    """A long cache whose values have a mean of one: what is left out of the sum does not average out."""
    d = 64
    K, q = rows((1, 1, N, d), dtype, 1), rows((1, n_q, 1, d), dtype, 2)
    V = (1 + 0.25 * rows((1, 1, N, d), "f32", 3)).to(DT[dtype])
    scale = 1.0 / 8
    out = call(ctx, dtype, d, n_q, N, q, K, V, scale, False)
    i = torch.arange(n_q, device="cuda")
    for r0 in range(0, n_q, 10):
        sees = torch.arange(N, device="cuda") <= (N - n_q + i[r0:r0 + 10])[:, None]
        ref, p, absum, size = definition(q[0, r0:r0 + 10, 0], K[0, 0], V[0, 0], sees, scale)
        # a lane adds up every eighth weight at most (four of the 32 of a half block, the densest), a product's sum every
        # eighth term or fewer; then 64 slices and their lanes and waves
        chain = N / 8 + 200
        e = 2 * (d + 4) * 2.0 ** -24 * size + 2.0 ** -22 + chain * 2.0 ** -24 + chain * 2.0 ** -24
        if dtype == "f16":
            tol = 2.0 ** -11 * ref.abs() + (e + 2.0 ** -11) * absum + N * 2.0 ** -34 * p.amax(1, keepdim=True) * V.abs().max().double() + 2.0 ** -25
        else:
            tol = 2.0 ** -24 * ref.abs() + e * absum + 2.0 ** -126
        err = (out[0, r0:r0 + 10, 0].double() - ref).abs()
        assert (err <= tol).all(), f"{(err / tol).max().item():.2f} tolerances"
