"""A decode step over a budget (append, attention with weights, eviction of one slot and of several), and a drafted tree with
its append, captured into one graph: every replay against the eager calls, with eager work in between."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import DT, desc, i32, random_tree, rows

pytestmark = pytest.mark.gpu


class Cache:
    """A pool and all arrays of its steps at fixed addresses."""

    def __init__(self, dtype, B, H, G, d, budget, T, r):
        self.shape, self.ctx = (B, H, G, d, budget, T), ig.Context(0)
        N_cap = budget + T + 1
        self.one, self.many = desc(B, H, d, budget + 1, N_cap, dtype, 0.2, r=r), desc(B, H, d, N_cap, N_cap, dtype, 0.2, r=r)
        self.K, self.V = rows((B, H, N_cap, d), dtype, 1), rows((B, H, N_cap, d), dtype, 2)
        self.mass = torch.rand((B * H, N_cap), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
        self.born = torch.arange(N_cap, dtype=torch.int32, device="cuda").repeat(B * H, 1)
        self.idx = torch.stack([torch.arange(h % 2, h % 2 + 2 * r, 2) for h in range(H)]).int().cuda()
        self.slab = torch.empty(ig.ig_slab_bytes(self.many), dtype=torch.uint8, device="cuda")
        self.ctx.ig_slab_build(self.many, self.K, ig.IG_MEM_DEVICE, self.idx, self.slab)
        self.q, self.k, self.v = (torch.zeros((B, T, x, d), dtype=DT[dtype], device="cuda") for x in (H * G, H, H))
        self.q1, self.k1, self.v1 = (torch.zeros((B, 1, x, d), dtype=DT[dtype], device="cuda") for x in (H * G, H, H))
        self.out, self.tree_out = torch.zeros_like(self.q1), torch.zeros_like(self.q)
        self.bits = torch.tensor([random_tree(T, b) for b in range(B)], dtype=torch.int64, device="cuda")
        self.path = i32([list(range(T))] * B)
        self.n_append, self.full, self.one_more, self.pos, self.guard, self.sum = (i32([x] * B) for x in (3, budget, budget + 1, budget, 8, 0))
        self.ctx.ig_reserve_cache(self.many, G, T)
        torch.cuda.synchronize()

    def step(self):
        B, H, G, d, budget, T = self.shape
        c = self.ctx
        c.ig_append_rows(self.one, 1, self.k1, self.v1, None, None, self.full, self.pos, self.idx, self.slab, self.K, self.V, self.mass, self.born)
        c.ig_cache_attention(self.one, G, 1, self.q1, None, self.K, self.V, self.one_more, self.mass, self.out)
        c.ig_pool_evict(self.one, budget, self.one_more, self.mass, self.born, self.guard, self.idx, self.slab, self.K, self.V)
        c.ig_tree_attention(self.many, G, T, self.q, self.k, self.v, self.bits, None, self.K, self.V, self.full, self.tree_out)
        c.ig_append_rows(self.many, T, self.k, self.v, self.path, self.n_append, self.full, self.pos, self.idx, self.slab, self.K, self.V,
                         self.mass, self.born)
        torch.add(self.full, self.n_append, out=self.sum)
        c.ig_pool_evict(self.many, budget, self.sum, self.mass, self.born, self.guard, self.idx, self.slab, self.K, self.V)
        self.pos += 4
        self.guard += 4

    def feed(self, dtype, seed):
        for i, x in enumerate((self.q, self.k, self.v, self.q1, self.k1, self.v1)):
            x.copy_(rows(tuple(x.shape), dtype, seed * 10 + i))
        self.n_append.copy_(torch.arange(len(self.n_append), device="cuda") + seed % 3)

    def state(self):
        return dict(K=self.K, V=self.V, mass=self.mass, born=self.born, slab=self.slab, out=self.out, tree=self.tree_out)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("group,T", [(1, 12), (4, 40)])
def test_steps_over_a_budget_in_a_graph(dtype, group, T):
    shape = (dtype, 3, 4, group, 64, 700, T, 19)
    captured, eager = Cache(*shape), Cache(*shape)
    held = captured.ctx.ig_workspace_bytes()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            captured.step()
    for seed in range(1, 6):
        captured.feed(dtype, seed)
        eager.feed(dtype, seed)
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for (name, a), b in zip(captured.state().items(), eager.state().values()):
            assert torch.equal(a, b), f"{name} after replay {seed}"
    assert captured.ctx.ig_workspace_bytes() == held
    captured.ctx.close()
    eager.ctx.close()
