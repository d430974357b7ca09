"""ig_pool_evict where as many slots are protected as may stay, or more: they still rank by weight among themselves."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import desc, i32, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def ranked(arrays, mass, born, kv, H, keep, protect):
    """The rule as it is documented: protection, the larger weight with NaN smallest, the lower slot."""
    for i in range(mass.shape[0]):
        n = kv[i // H]
        if n <= keep:
            continue
        m = mass[i, :n].astype(np.float64)
        nan = np.isnan(m)
        order = np.lexsort((np.arange(n), -np.where(nan, 0.0, m), nan, born[i, :n] < protect[i // H]))
        stay = np.sort(order[:keep])
        src, dst = stay[stay >= keep], np.setdiff1d(np.arange(keep), stay)
        for a in arrays:
            a[i, dst] = a[i, src]


def weights(kind, shape, rng):
    if kind == "ties":
        return rng.integers(0, 3, shape).astype(np.float32)
    m = rng.standard_normal(shape).astype(np.float32)
    if kind == "odd":
        for value, share in ((np.nan, 0.3), (np.inf, 0.2), (-np.inf, 0.2), (-0.0, 0.1), (0.0, 0.1)):
            m[rng.random(shape) < share] = value
    return m


# (N, keep, kv_len): one slot a pool, few, many; keys in registers of 512 and 1024 threads, and read again
SHAPES = [(2, 1, None), (65, 64, [65, 64]), (5000, 4999, None), (65, 55, [65, 60]), (300, 100, [300, 250]), (4096, 500, None),
          (5000, 2500, [5000, 2600]), (33000, 6000, None), (33000, 32990, [33000, 32995])]


@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
@pytest.mark.parametrize("over", [-1, 0, 1, 3, None], ids=lambda o: "all" if o is None else f"keep{o:+d}")
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{s[0]}to{s[1]}" for s in SHAPES])
def test_as_many_protected_as_stay(ctx, shape, over, kind):
    """`over` more protected than may stay, or all of them, scattered over the slots."""
    N, keep, kv = shape
    B, H, d, N_cap = 2, 2, 32, N + 3
    rng = np.random.default_rng(N * 7 + keep)
    K, V = rows((B, H, N_cap, d), "f16", 1), rows((B, H, N_cap, d), "f16", 2)
    lens = kv or [N] * B
    safe = [n if over is None else min(n, max(0, keep + over)) for n in lens]
    mass0 = weights(kind, (B * H, N_cap), rng)
    born0 = np.empty((B * H, N_cap), np.int32)
    for i in range(B * H):
        n = lens[i // H]
        born0[i, :n] = rng.permutation(n)
        born0[i, n:] = 1 << 30                     # slots behind the valid ones never count
    protect = [n - s for n, s in zip(lens, safe)]
    mass, born = torch.from_numpy(mass0).cuda(), torch.from_numpy(born0).cuda()
    state = [mass0.view(np.int32).copy(), born0.copy(), *(x.cpu().numpy().reshape(B * H, N_cap, d) for x in (K, V))]
    ranked(state, mass0, born0.copy(), lens, H, keep, protect)
    ctx.ig_pool_evict(desc(B, H, d, N, N_cap, "f16"), keep, i32(kv), mass, born, i32(protect), None, None, K, V)
    torch.cuda.synchronize()
    got = [mass.cpu().numpy().view(np.int32), born.cpu().numpy(), *(x.cpu().numpy().reshape(B * H, N_cap, d) for x in (K, V))]
    for name, a, b in zip(("mass", "born", "K", "V"), got, state):
        assert np.array_equal(a, b), name
