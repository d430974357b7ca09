"""ig_pool_evict and ig_append_rows against plain array operations, and the calls over a whole pool together."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import check_attention, desc, i32, random_tree, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def plain_evict(arrays, mass, born, kv, H, keep, protect):
    """The rule, pool by pool; arrays are numpy [B*H, N_cap, ..] that move along."""
    for i in range(mass.shape[0]):
        n = kv[i // H]
        if n <= keep:
            continue
        m = mass[i, :n].astype(np.float64)
        m[np.isnan(m)] = -np.inf
        lowest = np.isnan(mass[i, :n])
        safe = born[i, :n] >= protect[i // H] if protect is not None else np.zeros(n, bool)
        order = np.lexsort((np.arange(n), -m, lowest & ~safe, ~safe))
        stay = np.sort(order[:keep])
        src = stay[stay >= keep]
        dst = np.setdiff1d(np.arange(keep), stay)
        for a in arrays:
            a[i, dst] = a[i, src]


def make_pools(B, H, d, N_cap, dtype, seed):
    return rows((B, H, N_cap, d), dtype, seed), rows((B, H, N_cap, d), dtype, seed + 1)


def slab_rows(slab, ds):
    """The slab's entries as [B*H, slots, r]."""
    tile = 512 if ds.dtype == ig.IG_F16 else 256
    t = slab.view(torch.float16 if ds.dtype == ig.IG_F16 else torch.float32).view(ds.B * ds.H, -1, ds.r, tile)
    return t.transpose(2, 3).reshape(ds.B * ds.H, -1, ds.r)


def make_slab(ctx, ds, K, idx):
    slab = torch.empty(ig.ig_slab_bytes(ds), dtype=torch.uint8, device="cuda")
    ctx.ig_slab_build(ds, K, ig.IG_MEM_DEVICE, idx, slab)
    return slab


def weights(kind, BH, N_cap, rng):
    if kind == "random":
        return rng.exponential(size=(BH, N_cap)).astype(np.float32)
    if kind == "ties":
        return rng.integers(0, 3, (BH, N_cap)).astype(np.float32)
    if kind == "equal":
        return np.full((BH, N_cap), 0.5, np.float32)
    m = rng.standard_normal((BH, N_cap)).astype(np.float32)
    m[rng.random((BH, N_cap)) < 0.3] = np.nan
    m[rng.random((BH, N_cap)) < 0.1] = np.inf
    m[rng.random((BH, N_cap)) < 0.1] = -np.inf
    m[rng.random((BH, N_cap)) < 0.1] = -0.0
    m[rng.random((BH, N_cap)) < 0.1] = 0.0
    return m


# (B, H, d, N, N_cap, keep, kv_len)
EVICT = [
    (1, 1, 64, 2, 2, 1, None),
    (2, 3, 128, 65, 70, 64, None),
    (2, 3, 128, 65, 70, 64, [65, 40]),
    (3, 2, 64, 300, 300, 100, [300, 100, 101]),
    (2, 2, 96, 1000, 1003, 17, None),
    (2, 2, 32, 5000, 5001, 2500, [5000, 3333]),
    (1, 2, 64, 5000, 5000, 4999, None),
    (1, 2, 64, 33000, 33000, 6000, None),
    (1, 2, 64, 33000, 33000, 32990, [33000]),
    (2, 2, 64, 40, 40, 50, None),
    (1, 2, 512, 200, 200, 100, None),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("shape", EVICT, ids=[f"{s[3]}to{s[5]}d{s[2]}" for s in EVICT])
@pytest.mark.parametrize("guarded", [False, True])
def test_evict(ctx, dtype, kind, shape, guarded):
    B, H, d, N, N_cap, keep, kv = shape
    if d == 512 and dtype == "f32":
        d = 256
    rng = np.random.default_rng(N + keep)
    K, V = make_pools(B, H, d, N_cap, dtype, N)
    mass0 = weights(kind, B * H, N_cap, rng)
    born0 = np.stack([rng.permutation(N_cap) for _ in range(B * H)]).astype(np.int32)
    protect = [N_cap - keep // 2] * B if guarded else None
    mass, born = torch.from_numpy(mass0).cuda(), torch.from_numpy(born0).cuda()
    Kr, Vr = K.cpu().numpy().reshape(B * H, N_cap, d), V.cpu().numpy().reshape(B * H, N_cap, d)
    ctx.ig_pool_evict(desc(B, H, d, N, N_cap, dtype), keep, i32(kv), mass, born, i32(protect), None, None, K, V)
    torch.cuda.synchronize()
    state = [mass0.view(np.int32).copy(), born0.copy(), Kr, Vr]
    plain_evict(state, mass0, born0, kv or [N] * B, H, keep, protect)
    got = [mass.cpu().numpy().view(np.int32), born.cpu().numpy(), K.cpu().numpy().reshape(B * H, N_cap, d),
           V.cpu().numpy().reshape(B * H, N_cap, d)]
    for name, a, b in zip(("mass", "born", "K", "V"), got, state):
        assert np.array_equal(a, b), name


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("N,keep", [(601, 600), (1100, 300)])
def test_evict_moves_the_slab(ctx, dtype, N, keep):
    B, H, d, r, N_cap = 2, 3, 64, 19, 1200
    ds = desc(B, H, d, N, N_cap, dtype, r=r)
    K, V = make_pools(B, H, d, N_cap, dtype, 3)
    idx = torch.stack([torch.randperm(d, generator=torch.Generator().manual_seed(h))[:r].sort().values for h in range(H)]).int().cuda()
    slab = make_slab(ctx, ds, K, idx)
    mass = torch.rand((B * H, N_cap), device="cuda")
    ctx.ig_pool_evict(ds, keep, None, mass, None, None, idx, slab, K, V)
    after = make_slab(ctx, ds, K, idx)
    torch.cuda.synchronize()
    assert torch.equal(slab_rows(slab, ds)[:, :keep], slab_rows(after, ds)[:, :keep])


# (B, H, d, n_rows, N, N_cap, path, n_append, kv_len)
APPEND = [
    (1, 1, 64, 1, 0, 4, None, None, None),
    (2, 3, 128, 5, 7, 20, None, None, None),
    (3, 2, 96, 63, 100, 200, True, [5, 0, 63], [100, 3, 50]),
    (2, 2, 64, 64, 100, 110, True, [64, 2], [100, 0]),          # past the capacity: skipped
    (2, 2, 32, 700, 0, 1000, None, [700, 333], [0, 500]),
    (2, 1, 256, 70, 10, 100, None, [900, -3], [200, -7]),       # lengths outside their range
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("shape", APPEND, ids=[f"{s[3]}at{s[4]}d{s[2]}" for s in APPEND])
@pytest.mark.parametrize("with_slab", [False, True])
def test_append_rows(ctx, dtype, shape, with_slab):
    B, H, d, n_rows, N, N_cap, path, n_append, kv = shape
    rng = np.random.default_rng(n_rows)
    r = 7
    ds = desc(B, H, d, N, N_cap, dtype, r=r)
    K, V = make_pools(B, H, d, N_cap, dtype, 1)
    kr, vr = rows((B, n_rows, H, d), dtype, 5), rows((B, n_rows, H, d), dtype, 6)
    p = rng.integers(-2, n_rows + 2, (B, n_rows)).astype(np.int32) if path else None
    pos = rng.integers(0, 1000, B).astype(np.int32) if with_slab else None
    mass, born = torch.rand((B * H, N_cap), device="cuda"), torch.zeros((B * H, N_cap), dtype=torch.int32, device="cuda")
    idx = torch.stack([torch.randperm(d)[:r].sort().values for _ in range(H)]).int().cuda() if with_slab else None
    full = desc(B, H, d, N_cap, N_cap, dtype, r=r)
    slab = make_slab(ctx, full, K, idx) if with_slab else None
    want = [x.clone() for x in (K, V, mass.view(B, H, N_cap), born.view(B, H, N_cap))]
    for b in range(B):
        start = min(max(kv[b], 0), N_cap) if kv else N
        for j in range(min(max(n_append[b], 0), n_rows) if n_append else n_rows):
            if start + j >= N_cap:
                break
            src = min(max(int(p[b, j]), 0), n_rows - 1) if path else j
            want[0][b, :, start + j], want[1][b, :, start + j] = kr[b, src], vr[b, src]
            want[2][b, :, start + j] = 0
            want[3][b, :, start + j] = (int(pos[b]) if pos is not None else start) + j
    ctx.ig_append_rows(ds, n_rows, kr, vr, i32(p.tolist()) if path else None, i32(n_append), i32(kv),
                       i32(pos.tolist()) if pos is not None else None, idx, slab, K, V, mass, born)
    torch.cuda.synchronize()
    for name, a, b in zip(("K", "V", "mass", "born"), (K, V, mass.view(B, H, N_cap), born.view(B, H, N_cap)), want):
        assert torch.equal(a, b), name
    if with_slab:
        assert torch.equal(slab, make_slab(ctx, full, K, idx))


def test_append_of_one_row_is_append_token(ctx):
    B, H, d, r, N, N_cap = 2, 3, 64, 9, 40, 50
    ds = desc(B, H, d, N, N_cap, "f16", r=r)
    idx = torch.stack([torch.randperm(d)[:r].sort().values for _ in range(H)]).int().cuda()
    K, V = make_pools(B, H, d, N_cap, "f16", 1)
    slab = make_slab(ctx, ds, K, idx)
    k, v = rows((B, H, d), "f16", 2), rows((B, H, d), "f16", 3)
    K2, V2, slab2 = K.clone(), V.clone(), slab.clone()
    ctx.ig_append_token(ds, k, v, idx, slab, K, V, ig.IG_MEM_DEVICE)
    ctx.ig_append_rows(ds, 1, k, v, None, None, None, None, idx, slab2, K2, V2)
    torch.cuda.synchronize()
    assert torch.equal(K, K2) and torch.equal(V, V2) and torch.equal(slab, slab2)


def test_refusals(ctx):
    B, H, d, N = 2, 2, 64, 16
    ds = desc(B, H, d, N, N, "f16")
    K, V = make_pools(B, H, d, N, "f16", 1)
    K0 = K.clone()
    kr = rows((B, 4, H, d), "f16", 2)
    mass, born = torch.rand((B * H, N), device="cuda"), torch.zeros((B * H, N), dtype=torch.int32, device="cuda")
    guard = i32([0, 0])

    def refuse(code, f, *args):
        with pytest.raises(ig.IgError) as e:
            f(*args)
        assert e.value.code == code

    evict = lambda code, ds=ds, keep=8, mass=mass, born=born, guard=guard, idx=None, slab=None, K=K, V=V: refuse(   # noqa: E731
        code, ctx.ig_pool_evict, ds, keep, None, mass, born, guard, idx, slab, K, V)
    evict(ig.IG_ESHAPE, keep=0)
    evict(ig.IG_EINVAL, mass=None)
    evict(ig.IG_EINVAL, K=None)
    evict(ig.IG_EINVAL, V=None)
    evict(ig.IG_EINVAL, born=None)
    evict(ig.IG_EINVAL, slab=kr)
    evict(ig.IG_EINVAL, K=K.data_ptr() + 2)
    evict(ig.IG_ESHAPE, ds=desc(B, H, 60, N, N, "f16"))
    evict(ig.IG_ESHAPE, ds=desc(B, H, d, N, N - 1, "f16"))
    append = lambda code, ds=ds, n=4, k=kr, v=kr, idx=None, slab=None, K=K, V=V: refuse(   # noqa: E731
        code, ctx.ig_append_rows, ds, n, k, v, None, None, None, None, idx, slab, K, V)
    append(ig.IG_ESHAPE, n=0)
    for gone in ("k", "v", "K", "V"):
        append(ig.IG_EINVAL, **{gone: None})
    append(ig.IG_EINVAL, slab=kr)
    append(ig.IG_EINVAL, k=kr.data_ptr() + 8)
    append(ig.IG_EINVAL, k=K.data_ptr() + 16)
    append(ig.IG_EINVAL, v=V)
    append(ig.IG_ESHAPE, ds=desc(B, H, d, -1, N, "f16"))
    refuse(ig.IG_ESHAPE, ctx.ig_reserve_cache, ds, 0, 1)
    refuse(ig.IG_ESHAPE, ctx.ig_reserve_cache, ds, 1, 0)
    torch.cuda.synchronize()
    assert torch.equal(K, K0)


def test_profile_names_the_launches(ctx):
    B, H, d, N = 1, 2, 64, 300
    K, V = make_pools(B, H, d, N, "f16", 1)
    q, mass = rows((B, 1, H, d), "f16", 2), torch.rand((B * H, N), device="cuda")
    ds = desc(B, H, d, N, N, "f16")
    ctx.ig_profile_begin()
    ctx.ig_cache_attention(ds, 1, 1, q, None, K, V, None, mass, torch.empty_like(q))
    ctx.ig_pool_evict(ds, 100, None, mass, None, None, None, None, K, V)
    ctx.ig_profile_end()
    for which, launches in ((ig.IG_K_CACHE, 2), (ig.IG_K_EVICT, 2)):
        ms, n = ctx.ig_profile_read(which)
        assert n == launches and ms > 0


def test_budgeted_decoding_and_drafting(ctx):
    """The calls as they are used together, with a slab beside: a prompt with weights, the eviction to the budget,
    decode steps (append, attend with weights, evict by one), a drafted tree over the pool, its accepted path, and
    an eviction of what that left too much.  Every attention is compared with its definition over the pool as it
    is, every move with the plain rule."""
    B, H, G, d, r, dtype = 2, 2, 2, 64, 19, "f16"
    P, budget, recent, T = 150, 48, 16, 12
    N_cap = P + 8
    scale = 0.2
    ds = desc(B, H, d, P, N_cap, dtype, scale, r=r)
    idx = torch.stack([torch.arange(h, h + 3 * r, 3) for h in range(H)]).int().cuda()
    K, V = torch.zeros((B, H, N_cap, d), dtype=torch.float16, device="cuda"), torch.zeros((B, H, N_cap, d), dtype=torch.float16, device="cuda")
    mass, born = torch.zeros((B * H, N_cap), device="cuda"), torch.zeros((B * H, N_cap), dtype=torch.int32, device="cuda")
    slab = make_slab(ctx, desc(B, H, d, N_cap, N_cap, dtype, r=r), K, idx)
    prompt = [P, 97]
    pos = torch.tensor(prompt, dtype=torch.int32, device="cuda")       # the next token's position

    def attend(n_q, nq, kv, seed):
        q = rows((B, n_q, H * G, d), dtype, seed)
        out = torch.zeros_like(q)
        m0, o0 = mass.clone(), out.clone()
        ctx.ig_cache_attention(ds, G, n_q, q, i32(nq), K, V, i32(kv), mass, out)
        torch.cuda.synchronize()
        check_attention(q, K, V, kv, nq, G, float(np.float32(scale)), dtype, out, o0, mass, m0)

    def evict(kv):
        guard = pos - recent
        state = [x.cpu().numpy().copy() for x in (mass, born, K.view(B * H, N_cap, d), V.view(B * H, N_cap, d))]
        plain_evict(state, state[0].copy(), state[1].copy(), kv, H, budget, guard.tolist())
        ctx.ig_pool_evict(ds, budget, i32(kv), mass, born, guard, idx, slab, K, V)
        torch.cuda.synchronize()
        for a, b in zip((mass, born, K.view(B * H, N_cap, d), V.view(B * H, N_cap, d)), state):
            assert np.array_equal(a.cpu().numpy(), b)
        return [min(n, budget) for n in kv]

    def slab_matches(kv):
        whole = slab_rows(make_slab(ctx, desc(B, H, d, N_cap, N_cap, dtype, r=r), K, idx), ds)
        for b, n in enumerate(kv):
            assert torch.equal(slab_rows(slab, ds)[b * H:b * H + H, :n], whole[b * H:b * H + H, :n])

    k, v = rows((B, P, H, d), dtype, 1), rows((B, P, H, d), dtype, 2)
    ctx.ig_append_rows(ds, P, k, v, None, i32(prompt), i32([0, 0]), i32([0, 0]), idx, slab, K, V, mass, born)
    kv = list(prompt)
    attend(P, prompt, kv, 3)
    total = mass.view(B, H, N_cap).sum(2).double()
    # every query row's weights add up to one; each of the sums has at most 300 float32 roundings
    assert ((total - torch.tensor(prompt, device="cuda")[:, None] * G).abs() <= total * 300 * 2.0 ** -24 * 4).all()
    kv = evict(kv)
    slab_matches(kv)
    for step in range(3):
        k, v = rows((B, 1, H, d), dtype, 10 + step), rows((B, 1, H, d), dtype, 20 + step)
        ctx.ig_append_rows(ds, 1, k, v, None, None, i32(kv), pos, idx, slab, K, V, mass, born)
        pos += 1
        kv = [n + 1 for n in kv]
        attend(1, [1, 1], kv, 30 + step)
        kv = evict(kv)
        slab_matches(kv)
    tree = [random_tree(T, b) for b in range(B)]
    q, kt, vt = rows((B, T, H * G, d), dtype, 40), rows((B, T, H, d), dtype, 41), rows((B, T, H, d), dtype, 42)
    out = torch.zeros_like(q)
    o0 = out.clone()
    bits = torch.tensor(tree, dtype=torch.int64, device="cuda")
    ctx.ig_tree_attention(ds, G, T, q, kt, vt, bits, None, K, V, i32(kv), out)
    torch.cuda.synchronize()
    check_attention(q, K, V, kv, [T] * B, G, float(np.float32(scale)), dtype, out, o0, tree=(kt, vt, tree))
    # the accepted path: the ancestors of the last node, root first
    paths = [[j for j in range(T) if tree[b][T - 1] >> j & 1] for b in range(B)]
    path = i32([p + [0] * (T - len(p)) for p in paths])
    ctx.ig_append_rows(ds, T, kt, vt, path, i32([len(p) for p in paths]), i32(kv), pos, idx, slab, K, V, mass, born)
    torch.cuda.synchronize()
    for b, p in enumerate(paths):
        assert torch.equal(K[b, :, kv[b]:kv[b] + len(p)], kt[b, p].transpose(0, 1))
    pos += i32([len(p) for p in paths])
    kv = [n + len(p) for n, p in zip(kv, paths)]
    slab_matches(kv)
    attend(1, [1, 1], kv, 50)
    kv = evict(kv)
    slab_matches(kv)
    assert kv == [budget] * B
