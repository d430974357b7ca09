"""What the calls over a whole pool take and refuse: descriptors, arrays that overlap, sizes past a launch."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import SENTINEL, desc, i32, pools, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def refused(code, f, *args):
    with pytest.raises(ig.IgError) as e:
        f(*args)
    assert e.value.code == code, e.value


@pytest.mark.parametrize("odd", [dict(r=0), dict(r=-3), dict(r=300), dict(alpha=-1.0), dict(alpha=math.nan), dict(rope=7),
                                 dict(rope=1, rope_theta=0.0)], ids=str)
def test_fields_that_are_not_used_may_hold_anything(ctx, odd):
    """r without a slab, alpha and rope: the same results as with ordinary ones."""
    B, H, d, N, N_cap = 2, 2, 64, 40, 48
    results = []
    for fields in ({}, odd):
        ds = desc(B, H, d, N, N_cap, "f16", 0.125)
        for name, value in fields.items():
            setattr(ds, name, value)
        K, V = pools(B, H, d, N_cap, "f16", [N] * B, 1)
        q, kt, vt = rows((B, 3, H, d), "f16", 2), rows((B, 3, H, d), "f16", 3), rows((B, 3, H, d), "f16", 4)
        bits = torch.tensor([[1, 3, 5]] * B, dtype=torch.int64, device="cuda")
        mass, born = torch.zeros((B * H, N_cap), device="cuda"), torch.zeros((B * H, N_cap), dtype=torch.int32, device="cuda")
        out, tree = torch.zeros_like(q), torch.zeros_like(q)
        ctx.ig_reserve_cache(ds, 1, 3)
        ctx.ig_cache_attention(ds, 1, 3, q, None, K, V, None, mass, out)
        ctx.ig_tree_attention(ds, 1, 3, q, kt, vt, bits, None, K, V, None, tree)
        ctx.ig_append_rows(ds, 3, kt, vt, None, None, None, None, None, None, K, V, None, born)
        ctx.ig_pool_evict(ds, 20, None, mass, born, None, None, None, K, V)
        torch.cuda.synchronize()
        results.append([out, tree, mass, born, K.nan_to_num(), V.nan_to_num()])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("r", [0, 65, -1])
def test_a_slab_needs_its_channels(ctx, r):
    ds = desc(1, 1, 64, 8, 16, "f16", r=r)
    K, V = pools(1, 1, 64, 16, "f16", [16], 1)
    x = rows((1, 1, 1, 64), "f16", 2)
    idx, slab, mass = i32([0]), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda"), torch.zeros((1, 16), device="cuda")
    refused(ig.IG_ESHAPE, ctx.ig_append_rows, ds, 1, x, x, None, None, None, None, idx, slab, K, V)
    refused(ig.IG_ESHAPE, ctx.ig_pool_evict, ds, 4, None, mass, None, None, idx, slab, K, V)


def test_out_apart_from_every_input(ctx):
    """The masks, the lengths and the weights too."""
    B, H, d, N = 2, 2, 64, 16
    ds = desc(B, H, d, N, N, "f16")
    K, V = pools(B, H, d, N, "f16", [N] * B, 1)
    q, kt = rows((B, 4, H, d), "f16", 2), rows((B, 4, H, d), "f16", 3)
    out = torch.full_like(q, SENTINEL)
    inside = out.view(-1)[64:]                     # 16-byte aligned, and in the output's last bytes
    ends = out.view(-1)[-8:]
    bits = torch.zeros((B, 4), dtype=torch.int64, device="cuda")
    lens, mass = i32([1, 1]), torch.zeros((B * H, N), device="cuda")
    for at in (inside, ends, out.data_ptr() - 4):
        refused(ig.IG_EINVAL, ctx.ig_cache_attention, ds, 1, 4, q, at, K, V, lens, mass, out)
        refused(ig.IG_EINVAL, ctx.ig_cache_attention, ds, 1, 4, q, lens, K, V, at, mass, out)
        refused(ig.IG_EINVAL, ctx.ig_cache_attention, ds, 1, 4, q, lens, K, V, lens, at, out)
        refused(ig.IG_EINVAL, ctx.ig_tree_attention, ds, 1, 4, q, kt, kt, bits, at, K, V, lens, out)
        refused(ig.IG_EINVAL, ctx.ig_tree_attention, ds, 1, 4, q, kt, kt, bits, lens, K, V, at, out)
    for at in (inside, ends, out.data_ptr() - 8):
        refused(ig.IG_EINVAL, ctx.ig_tree_attention, ds, 1, 4, q, kt, kt, at, lens, K, V, lens, out)
    torch.cuda.synchronize()
    assert (out == SENTINEL).all()
    # next to each other is apart
    both = torch.zeros(out.numel() * 2 + B * H * N * 4, dtype=torch.uint8, device="cuda")
    o, m = both[:out.numel() * 2], both[out.numel() * 2:]
    ctx.ig_cache_attention(ds, 1, 4, q, None, K, V, None, m, o)
    torch.cuda.synchronize()


def test_more_than_a_launch_takes(ctx):
    """Refused for its size before anything else: every call here also has an argument that is refused later."""
    x = torch.zeros(1 << 12, dtype=torch.float16, device="cuda")
    bad = x.data_ptr() + 2
    # 2^23 pools: too many for a selection's 512 threads each, not for 256
    refused(ig.IG_ESHAPE, ctx.ig_pool_evict, desc(1 << 12, 1 << 11, 64, 3, 3, "f16"), 1, None, x, None, None, None, None, bad, x)
    refused(ig.IG_EINVAL, ctx.ig_pool_evict, desc(1 << 12, 1 << 11, 64, 3, 3, "f16"), 2, None, x, None, None, None, None, bad, x)
    refused(ig.IG_EINVAL, ctx.ig_cache_attention, desc(1 << 12, 1 << 11, 64, 1, 1, "f16"), 1, 1, bad, None, x, x, None, None, x)
    refused(ig.IG_EINVAL, ctx.ig_append_rows, desc(1 << 12, 1 << 11, 64, 1, 1, "f16"), 1, bad, x, None, None, None, None, None, None, x, x)
    # 2^29 float32 slots in blocks of 32 keys: 2^24 workgroups; out is q, which is looked at afterwards
    refused(ig.IG_ESHAPE, ctx.ig_cache_attention, desc(1, 1 << 9, 32, 1 << 20, 1 << 20, "f32"), 1, 2, x, None, x, x, None, x, x)
    refused(ig.IG_EINVAL, ctx.ig_cache_attention, desc(1, 1 << 9, 32, 1 << 20, 1 << 20, "f32"), 1, 2, x, None, x, x, None, None, x)
    refused(ig.IG_EINVAL, ctx.ig_cache_attention, desc(1, 1 << 9, 32, 1 << 20, 1 << 20, "f32"), 1, 1, x, None, x, x, None, x, x)
    # 2^31 slots, half of them kept: 2^24 blocks of 64 rows that could move
    refused(ig.IG_ESHAPE, ctx.ig_pool_evict, desc(1, 1 << 9, 8, 1 << 22, 1 << 22, "f16"), 1 << 21, None, x, None, None, None, None, bad, x)
    refused(ig.IG_EINVAL, ctx.ig_pool_evict, desc(1, 1 << 9, 8, 1 << 22, 1 << 22, "f16"), 1 << 20, None, x, None, None, None, None, bad, x)
