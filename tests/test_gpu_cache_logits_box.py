"""The weights of single-token calls, whose logits pass between a wave's lanes: waves that fill
their part of LDS several times over, exactly once, and not at all."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2406_19707_amd as ig
from ig_cache import run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = ig.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("group,N", [(1, 12800), (3, 5001), (7, 3333), (16, 4100)])
def test_logits_of_every_tile(ctx, dtype, d, group, N):
    """So many pools that each has one slice or a few, and a wave many tiles of it."""
    B = 64 if group == 1 else 24
    kv = [N - 17 * b for b in range(B)]
    run_attention(ctx, dtype, d, B, 8, group, 1, N, N + 1, kv, None, seed=group)
