"""Trees of drafted tokens whose queries, keys and values have nothing in common, over more sequences than a wave has lanes,
and with nodes that none sees."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import SENTINEL, check_attention, desc, i32, pools, random_tree, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


def run_tree_apart(ctx, dtype, d, B, H, group, T, N, kv, nt, visible, scale=0.2, seed=11, bad_nodes=()):
    """ig_tree_attention with queries, keys and values that have nothing in common."""
    lens, tlens = kv or [N] * B, nt or [T] * B
    K, V = pools(B, H, d, N + 3, dtype, lens, seed)
    q, kt, vt = rows((B, T, H * group, d), dtype, seed + 1), rows((B, T, H, d), dtype, seed + 2), rows((B, T, H, d), dtype, seed + 3)
    assert not torch.equal(kt, vt)
    for b, m in enumerate(tlens):
        q[b, m:], kt[b, m:], vt[b, m:] = float("nan"), float("nan"), float("inf")
    clean = kt.clone(), vt.clone()
    for j in bad_nodes:
        kt[:, j], vt[:, j] = float("inf"), float("nan")
    out = torch.full_like(q, SENTINEL)
    before = out.clone()
    bits = torch.tensor([[v - (1 << 64) if v >> 63 else v for v in row] for row in visible], dtype=torch.int64, device="cuda")
    ctx.ig_tree_attention(desc(B, H, d, N, N + 3, dtype, scale), group, T, q, kt, vt, bits, i32(nt), K, V, i32(kv), out)
    torch.cuda.synchronize()
    check_attention(q, K, V, lens, tlens, group, float(torch.tensor(scale, dtype=torch.float32)), dtype, out, before,
                    tree=(*clean, visible))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("group,T", [(1, 9), (1, 40), (5, 30)])
@pytest.mark.parametrize("kind", ["ragged", "one long", "empty"])
def test_trees_over_many_ragged_sequences(ctx, dtype, group, T, kind):
    B, N = 70, 1500
    kv = {"ragged": [(b * 37 % 64) * 23 for b in range(B)], "one long": [N if b == 66 else 1 for b in range(B)], "empty": [0] * B}[kind]
    run_tree_apart(ctx, dtype, 64, B, 1, group, T, N, kv, [T - b % 7 for b in range(B)], [random_tree(T, b) for b in range(B)])


# (B, H, group, T, N, kv_len, nodes)
TREES = [
    (1, 1, 1, 1, 0, [0], None),
    (2, 2, 1, 13, 70, None, None),
    (2, 3, 4, 64, 200, [200, 31], [64, 33]),           # four waves, or eight with 256 rows
    (3, 1, 2, 33, 65, [0, 1, 65], [33, 5, 32]),
    (1, 2, 8, 63, 1025, None, None),
    (2, 2, 1, 48, 4096, [4000, 64], [48, 40]),
    (2, 1, 1, 17, 4096, [4000, 5], [1, 17]),
]


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("shape", TREES, ids=[f"{s[3]}over{s[4]}x{s[2]}" for s in TREES])
def test_trees_whose_keys_values_and_queries_differ(ctx, dtype, d, shape):
    B, H, group, T, N, kv, nt = shape
    run_tree_apart(ctx, dtype, d, B, H, group, T, N, kv, nt, [random_tree(T, d + b) for b in range(B)])


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("group", [1, 4])
def test_tree_masks_and_nodes_that_none_sees(ctx, dtype, group):
    T, full = 64, (1 << 64) - 1
    masks = [0 if i % 3 == 0 else (full if i % 3 == 1 else 1 << 63) for i in range(T)]
    unseen = [v & ~(1 << 7 | 1 << 39) for v in random_tree(T, 3)]
    for kv in ([0, 0], [37, 0], [130, 64]):
        run_tree_apart(ctx, dtype, 64, 2, 2, group, T, 130, kv, None, [masks] * 2)
        run_tree_apart(ctx, dtype, 64, 2, 2, group, T, 130, kv, None, [unseen, [0] * T], bad_nodes=(7, 39))
