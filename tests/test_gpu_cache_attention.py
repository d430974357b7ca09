"""ig_cache_attention and ig_tree_attention against their definition in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import SENTINEL, desc, i32, pools, random_tree, rows, run_attention, run_tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


# (B, H, group, n_q, N, spare slots, kv_len, q_len)
SHAPES = [
    (1, 1, 1, 1, 1, 0, None, None),
    (2, 3, 1, 1, 33, 5, None, None),
    (3, 2, 4, 1, 130, 1, [130, 1, 0], None),
    (2, 2, 8, 1, 517, 3, [17, 517], [1, 0]),
    (2, 2, 1, 5, 5, 0, None, None),
    (2, 1, 2, 17, 40, 9, [3, 40], [17, 16]),       # more queries than slots: the first see nothing
    (1, 2, 3, 63, 257, 0, None, None),
    (3, 2, 1, 65, 129, 2, [129, 65, 64], [65, 1, 0]),
    (1, 2, 1, 300, 300, 20, None, None),
    (2, 1, 4, 97, 1000, 0, [1000, 431], [97, 50]),
    (1, 1, 16, 1, 64, 0, None, None),
    (1, 2, 65, 1, 70, 0, None, None),              # more heads to a pool than the kept logits are for
    (2, 3, 1, 128, 640, 0, [640, 128], None),
    (2, 2, 2, 257, 513, 7, [513, 300], [257, 129]),
    (2, 2, 1, 2, 300, 0, [300, 0], None),
    (1, 2, 17, 1, 90, 3, None, None),
    (2, 1, 32, 1, 33, 0, [0, 33], None),
    (1, 1, 1, 33, 64, 0, None, None),
    (1, 1, 5, 26, 128, 0, None, None),             # 130 rows that mostly see the same
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{s[3]}of{s[4]}x{s[2]}" for s in SHAPES])
def test_cache_attention(ctx, dtype, d, shape):
    B, H, group, n_q, N, spare, kv, nq = shape
    run_attention(ctx, dtype, d, B, H, group, n_q, N, N + spare, kv, nq, seed=d + N)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n_q,N,scale", [(1, 100, -0.2), (1, 100, 0.0), (40, 90, -0.2), (40, 90, 0.0), (200, 260, -0.2),
                                         (200, 260, 0.0), (1, 100, 3.0), (200, 260, 3.0)])
def test_scale_of_any_sign(ctx, dtype, n_q, N, scale):
    run_attention(ctx, dtype, 64, 2, 2, 2, n_q, N, N, None, None, scale=scale)


@pytest.mark.parametrize("dtype,B,H,n_q,N", [("f16", 1, 2, 1, 20000), ("f32", 1, 1, 1, 9000), ("f16", 1, 1, 70, 12345),
                                             ("f16", 8, 16, 130, 200), ("f32", 4, 33, 129, 180), ("f16", 4, 64, 1, 700)])
def test_long_and_wide(ctx, dtype, B, H, n_q, N):
    run_attention(ctx, dtype, 128, B, H, 1, n_q, N, N + 3, None, None)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("group", [1, 40])
@pytest.mark.parametrize("kind", ["ragged", "one long", "empty", "full"])
def test_slices_of_many_ragged_sequences(ctx, dtype, group, kind):
    """More sequences than a wave has lanes, their slices dealt by length."""
    B, N = 70, 2500
    kv = {"ragged": [(b * 37 % 64) * 39 for b in range(B)], "one long": [N if b == 66 else 1 for b in range(B)],
          "empty": [0] * B, "full": [N] * B}[kind]
    run_attention(ctx, dtype, 64, B, 1, group, 1, N, N + 1, kv, [b % 5 and 1 for b in range(B)])


@pytest.mark.parametrize("n_q,N", [(1, 333), (100, 333)])
def test_without_weights_is_the_same(ctx, n_q, N):
    a = run_attention(ctx, "f16", 128, 2, 2, 2, n_q, N, N, None, None, with_mass=True)
    b = run_attention(ctx, "f16", 128, 2, 2, 2, n_q, N, N, None, None, with_mass=False)
    assert torch.equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
def test_row_blocks_and_key_blocks_in_pairs(ctx, d):
    """Calls large enough for workgroups to take two blocks each, an odd number of them."""
    run_attention(ctx, "f16", d, 8, 64, 1, 300, 513, 514, [513, 300, 1, 0, 257, 512, 400, 299], [300, 300, 1, 300, 0, 129, 300, 299])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n_q", [1, 5, 40])
def test_no_slots(ctx, dtype, n_q):
    """N = 0: every row that is there becomes zero, no weight changes."""
    run_attention(ctx, dtype, 64, 2, 2, 2, n_q, 0, 7, None, [n_q, 0])


def test_far_slots(ctx):
    """Byte offsets past 32 bits within a pool and across pools."""
    d, N_cap = 256, 4_300_000                     # 2.2 GB a pool of keys
    g = torch.Generator(device="cuda").manual_seed(3)
    K = torch.empty((1, 2, N_cap, d), dtype=torch.float16, device="cuda").normal_(generator=g)
    V = torch.empty_like(K).normal_(generator=g)
    q = rows((1, 1, 2, d), "f16", 4)
    out = torch.zeros_like(q)
    mass = torch.zeros((2, N_cap), device="cuda")
    scale = 1.0 / 16
    K[:, :, N_cap - 7] = q[0, 0].view(2, d) * 2   # one slot at the end that outweighs the rest
    ctx.ig_cache_attention(desc(1, 2, d, N_cap, N_cap, "f16", scale), 1, 1, q, None, K, V, None, mass, out)
    torch.cuda.synchronize()
    for h in range(2):
        s = (K[0, h].float() @ q[0, 0, h].float()).double() * scale
        p = torch.softmax(s, 0)
        ref = p.float() @ V[0, h].float()
        # float32 reference sums: a relative 1e-3 of the sum of |p v| (at most 5 here) covers both sides
        assert ((out[0, 0, h].float() - ref).abs() <= 5e-3).all()
        assert p[N_cap - 7] > 0.5 and abs(mass[h, N_cap - 7].item() - p[N_cap - 7].item()) <= 1e-3
        assert (mass[h].double() - p).abs().max() <= 1e-3


TREES = [
    (1, 1, 1, 1, 0, [0], None),
    (1, 1, 1, 1, 0, None, None),
    (2, 2, 1, 13, 70, None, None),
    (2, 3, 4, 64, 200, [200, 31], [64, 33]),
    (3, 1, 2, 33, 65, [0, 1, 65], [33, 0, 32]),
    (1, 2, 8, 63, 1025, None, None),
    (2, 1, 1, 17, 4096, [4000, 5], [1, 17]),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("shape", TREES, ids=[f"{s[3]}over{s[4]}x{s[2]}" for s in TREES])
def test_tree_attention(ctx, dtype, d, shape):
    B, H, group, T, N, kv, nt = shape
    run_tree(ctx, dtype, d, B, H, group, T, N, N + 2, kv, nt, [random_tree(T, d + b) for b in range(B)])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_tree_masks(ctx, dtype):
    """Nodes that see nothing (not even themselves), everything, or only the last node."""
    T = 64
    full = (1 << 64) - 1
    for kv in ([0, 0], [37, 0]):
        run_tree(ctx, dtype, 64, 2, 2, 1, T, 40, 40, kv, None,
                 [[0 if i % 3 == 0 else (full if i % 3 == 1 else 1 << 63) for i in range(T)]] * 2)


@pytest.mark.parametrize("dtype,group,d", [("f16", 1, 64), ("f16", 4, 64), ("f16", 3, 256), ("f32", 1, 128)])
@pytest.mark.parametrize("kv", [[45, 3], [0, 45]])
def test_nodes_that_none_sees_may_hold_anything(ctx, dtype, group, d, kv):
    T, N = 40, 45
    masks = [v & ~(1 << 7 | 1 << 39) for v in random_tree(T, 3)]
    for visible in ([masks, masks], [masks, [0] * T]):
        run_tree(ctx, dtype, d, 2, 2, group, T, N, N, kv, None, visible, bad_nodes=(7, 39))


def test_a_chain_is_a_chunk(ctx):
    """A tree that is a chain gives the chunk's attention over the same keys."""
    B, H, G, T, N, d = 2, 2, 2, 24, 150, 64
    K, V = pools(B, H, d, N + T, "f32", [N + T] * B, 5)
    q = rows((B, T, H * G, d), "f32", 6)
    one, two = torch.zeros_like(q), torch.zeros_like(q)
    ctx.ig_cache_attention(desc(B, H, d, N + T, N + T, "f32", 0.1), G, T, q, None, K, V, None, None, one)
    kt, vt = (x[:, :, N:].transpose(1, 2).contiguous() for x in (K, V))
    bits = torch.tensor([[(1 << (i + 1)) - 1 for i in range(T)]] * B, dtype=torch.int64, device="cuda")
    ctx.ig_tree_attention(desc(B, H, d, N, N + T, "f32", 0.1), G, T, q, kt, vt, bits, None, K, V, None, two)
    # two orders of the same float32 sums of 174 terms below 5 in size
    assert (one - two).abs().max() <= 174 * 2.0 ** -24 * 5 * 4


def test_refusals(ctx):
    B, H, d, N = 2, 2, 64, 16
    K, V = pools(B, H, d, N, "f16", [N] * B, 1)
    q = rows((B, 4, H, d), "f16", 2)
    kt, vt = rows((B, 4, H, d), "f16", 3), rows((B, 4, H, d), "f16", 4)
    bits = torch.zeros((B, 4), dtype=torch.int64, device="cuda")
    out = torch.full_like(q, SENTINEL)
    ds = desc(B, H, d, N, N, "f16")

    def attention(code, ds=ds, group=1, n_q=4, q=q, K=K, V=V, out=out):
        with pytest.raises(ig.IgError) as e:
            ctx.ig_cache_attention(ds, group, n_q, q, None, K, V, None, None, out)
        assert e.value.code == code

    def tree(code, ds=ds, group=1, T=4, q=q, kt=kt, vt=vt, bits=bits, K=K, V=V, out=out):
        with pytest.raises(ig.IgError) as e:
            ctx.ig_tree_attention(ds, group, T, q, kt, vt, bits, None, K, V, None, out)
        assert e.value.code == code

    for f in (attention, tree):
        for gone in ("q", "K", "V", "out"):
            f(ig.IG_EINVAL, **{gone: None})
            f(ig.IG_EINVAL, **{gone: q.data_ptr() + 2})
        f(ig.IG_ESHAPE, group=0)
        f(ig.IG_ESHAPE, ds=desc(B, H, 96, N, N, "f16"))
        f(ig.IG_ESHAPE, ds=desc(B, H, 512, N, N, "f16"))
        f(ig.IG_ESHAPE, ds=desc(0, H, d, N, N, "f16"))
        f(ig.IG_ESHAPE, ds=desc(B, H, d, N, N - 1, "f16"))
        f(ig.IG_ESHAPE, ds=desc(B, H, d, -1, N, "f16"))
        f(ig.IG_ESHAPE, group=1 << 30)
        f(ig.IG_EINVAL, ds=desc(B, H, d, N, N, "f16", float("nan")))
    attention(ig.IG_ESHAPE, n_q=0)
    attention(ig.IG_ESHAPE, n_q=1 << 30)
    tree(ig.IG_ESHAPE, T=0)
    tree(ig.IG_ESHAPE, T=65)
    for gone in ("kt", "vt", "bits"):
        tree(ig.IG_EINVAL, **{gone: None})
    bad = desc(B, H, d, N, N, "f16")
    bad.dtype = 5
    attention(ig.IG_EDTYPE, ds=bad)
    with pytest.raises(AssertionError):
        ctx.ig_cache_attention(ds, 1, 4, q.transpose(1, 2), None, K, V, None, None, out)
    attention(ig.IG_EINVAL, out=q)
    attention(ig.IG_EINVAL, out=K.data_ptr() + 16)
    tree(ig.IG_EINVAL, out=vt.data_ptr() + 32)
    tree(ig.IG_EINVAL, bits=bits.data_ptr() + 4)
    torch.cuda.synchronize()
    assert (out == SENTINEL).all()


def test_lengths_are_clamped(ctx):
    """Lengths outside their range act as the nearest one inside it."""
    B, H, d, N = 2, 2, 64, 50
    K, V = pools(B, H, d, N, "f32", [N] * B, 1)
    q = rows((B, 3, H, d), "f32", 2)
    outs = []
    for kv, nq in (([N + 100, -5], [9, 3]), ([N, 0], [3, 3])):
        out = torch.full_like(q, SENTINEL)
        ctx.ig_cache_attention(desc(B, H, d, N, N, "f32", 0.1), 1, 3, q, i32(nq), K, V, i32(kv), None, out)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and (outs[0][1] == 0).all()


@pytest.mark.parametrize("n_q,N", [(1, 900), (150, 700)])
def test_graph_replays(ctx, n_q, N):
    """Captured after ig_reserve_cache, replayed with eager work between, each replay against the eager call."""
    B, H, G, d = 2, 4, 2, 128
    c = ig.Context(0)
    ds = desc(B, H, d, N, N, "f16", 0.1)
    K, V = pools(B, H, d, N, "f16", [N] * B, 1)
    q = rows((B, n_q, H * G, d), "f16", 2)
    out, ref = torch.zeros_like(q), torch.zeros_like(q)
    mass, mref = torch.zeros((B * H, N), device="cuda"), torch.zeros((B * H, N), device="cuda")
    kv = i32([N, N - 100])
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            with pytest.raises(ig.IgError) as e:         # nothing reserved, nothing may be allocated
                c.ig_cache_attention(ds, G, n_q, q, None, K, V, kv, mass, out)
            assert e.value.code == ig.IG_EINVAL
    c.ig_reserve_cache(ds, G, n_q)
    held = c.ig_workspace_bytes()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            c.ig_cache_attention(ds, G, n_q, q, None, K, V, kv, mass, out)
    for step in range(4):
        q.copy_(rows(q.shape, "f16", 10 + step))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        ctx.ig_cache_attention(ds, G, n_q, q, None, K, V, kv, mref, ref)
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(mass, mref)
    assert c.ig_workspace_bytes() == held
    c.close()


def test_other_streams_and_contexts_at_once(ctx):
    """Two contexts on two streams give what one gives."""
    args = ("f16", 128, 4, 8, 1, 1, 2000, 2000, None, None)
    want = run_attention(ctx, *args)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = ig.Context(0)
        got = run_attention(other, *args)
        other.close()
    assert torch.equal(want, got)


def test_reserved_covers_smaller_calls():
    c = ig.Context(0)
    B, H, G, d, N = 1, 2, 2, 64, 3000
    ds = desc(B, H, d, 100, N, "f16", 0.1)
    c.ig_reserve_cache(ds, G, 100)
    held = c.ig_workspace_bytes()
    K, V = pools(B, H, d, N, "f16", [N], 1)
    q = rows((B, 100, H * G, d), "f16", 2)
    kt = rows((B, 64, H, d), "f16", 3)
    out, mass = torch.empty_like(q), torch.zeros((B * H, N), device="cuda")
    bits = torch.zeros((B, 64), dtype=torch.int64, device="cuda")
    for n in (1, 2, 7, 8, 9, 16, 31, 32, 33, 64, 100):
        for length in (1, 77, 1500, N):
            ds.N = length
            c.ig_cache_attention(ds, G, n, q, None, K, V, None, mass, out)
            if n <= 64:
                c.ig_tree_attention(ds, G, n, q, kt, kt, bits, None, K, V, None, out)
    for keep in (1, 100, 1500, N - 1):
        c.ig_pool_evict(ds, keep, None, mass, None, None, None, None, K, V)
    torch.cuda.synchronize()
    assert c.ig_workspace_bytes() == held
    c.close()
