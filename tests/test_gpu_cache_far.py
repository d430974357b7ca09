"""Slots whose bytes lie past 2^31 and 2^32 inside one pool: their weights one by one, and an output that they make alone."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import desc, rows

pytestmark = pytest.mark.gpu

D, N = 256, (1 << 23) + 70001                     # 512 bytes a row: slot 2^23 is at byte 2^32
SCALE = 1.0 / 16


@pytest.fixture(scope="module")
def cache():
    g = torch.Generator(device="cuda").manual_seed(3)
    K = torch.empty((1, 1, N, D), dtype=torch.float16, device="cuda").normal_(generator=g)
    V = torch.zeros_like(K)
    V[:, :, 1 << 23:].normal_(mean=1.0, std=0.25, generator=g)
    yield K, V
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n_q", [1, 40])
def test_far_slots(cache, n_q):
    K, V = cache
    ctx = ig.Context(0)
    q = rows((1, n_q, 1, D), "f16", 4)
    out, mass = torch.zeros_like(q), torch.zeros((1, N), device="cuda")
    ctx.ig_cache_attention(desc(1, 1, D, N, N, "f16", SCALE), 1, n_q, q, None, K, V, None, mass, out)
    torch.cuda.synchronize()
    ctx.close()
    Q, last = q[0, :, 0].double(), N - n_q + torch.arange(n_q, device="cuda")
    step = 1 << 18
    total = torch.zeros((n_q, 1), dtype=torch.float64, device="cuda")
    size = 0.0

    def logits(t0):
        t = torch.arange(t0, min(N, t0 + step), device="cuda")
        return torch.where(t <= last[:, None], Q @ K[0, 0, t0:t0 + step].double().T * SCALE, -torch.inf)

    for t0 in range(0, N, step):                   # (logits of normal rows of 256 channels over 16 stay below 10 in size)
        total += torch.exp(logits(t0)).sum(1, keepdim=True)
        size = max(size, (Q.abs() @ K[0, 0, t0:t0 + step].double().abs().T).max().item() * SCALE)
    # the sum in float32: 64 slices at least a pool's 32-token tiles long; a lane adds 8 terms of each of its turns at most, then
    # lanes, waves and slices; the weight itself as in ig_cache
    chain = N / 64 / 64 * 8 + 300
    e = 2 * (D + 4) * 2.0 ** -24 * size + 2.0 ** -22 + chain * 2.0 ** -24
    assert e < 5e-3
    ref, absum = torch.zeros((n_q, D), dtype=torch.float64, device="cuda"), torch.zeros((n_q, D), dtype=torch.float64, device="cuda")
    for t0 in range(0, N, step):
        p = torch.exp(logits(t0)) / total
        want = p.sum(0)
        err = (mass[0, t0:t0 + step].double() - want).abs()
        assert (err <= (e + (n_q + 4) * 2.0 ** -24) * want).all(), f"slot {t0 + int((err / want).argmax())}"
        v = V[0, 0, t0:t0 + step].double()
        ref += p @ v
        absum += p @ v.abs()
    # the output as in ig_cache; weights are rounded to half precision by 2^-11 of themselves, or by 2^-34 of the largest
    largest = torch.exp(torch.stack([logits(t0).amax(1) for t0 in range(0, N, step)]).amax(0))[:, None] / total
    tol = 2.0 ** -11 * ref.abs() + (e + chain * 2.0 ** -24 + 2.0 ** -11) * absum + 70001 * 2.0 ** -34 * largest * V.abs().max().double() + 2.0 ** -25
    assert (ref > 10 * tol).all()
    assert ((out[0, :, 0].double() - ref).abs() <= tol).all()


def test_far_rows_are_written_and_moved(cache):
    """Rows appended behind byte 2^32, which an eviction then moves to the holes below."""
    K, V = cache
    ctx = ig.Context(0)
    at, n = N - 20, 9
    k, v = rows((1, n, 1, D), "f16", 5), rows((1, n, 1, D), "f16", 6)
    mass = torch.ones((1, N), device="cuda")
    born = torch.arange(N, dtype=torch.int32, device="cuda").view(1, N)
    before = K[0, 0, at - 3:].clone()
    ctx.ig_append_rows(desc(1, 1, D, at, N, "f16"), n, k, v, None, None, None, torch.tensor([N], dtype=torch.int32, device="cuda"),
                       None, None, K, V, mass, born)
    torch.cuda.synchronize()
    assert torch.equal(K[0, 0, at:at + n], k[0, :, 0]) and torch.equal(V[0, 0, at:at + n], v[0, :, 0])
    assert torch.equal(K[0, 0, at - 3:at], before[:3]) and torch.equal(K[0, 0, at + n:], before[3 + n:])
    assert (mass[0, at:at + n] == 0).all() and torch.equal(born[0, at:at + n], N + torch.arange(n, dtype=torch.int32, device="cuda"))
    holes = torch.tensor([0, 5, 1000, (1 << 22) + 1, (1 << 23) + 3], device="cuda")
    mass[0, holes] = -1.0
    mass[0, at:at + n] = 2.0
    keep = at + n - len(holes)
    ctx.ig_pool_evict(desc(1, 1, D, at + n, N, "f16"), keep, None, mass, born, None, None, None, K, V)
    torch.cuda.synchronize()
    assert torch.equal(K[0, 0, holes], k[0, -5:, 0]) and torch.equal(V[0, 0, holes], v[0, -5:, 0])
    assert (mass[0, holes] == 2).all() and torch.equal(born[0, holes], N + 4 + torch.arange(5, dtype=torch.int32, device="cuda"))
    ctx.close()
