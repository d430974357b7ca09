"""Slices dealt to sequences of very different lengths: one long one among many short ones, which takes no more than it has
work for; and paired blocks at the head dimensions that are rarely met."""
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
@pytest.mark.parametrize("group,n_q", [(1, 1), (8, 1), (1, 40), (2, 130)])
@pytest.mark.parametrize("B,N,short", [(16, 9000, 64), (16, 9000, 0), (70, 2500, 1), (5, 4097, 127)])
def test_one_long_sequence(ctx, dtype, group, n_q, B, N, short):
    for long_one in (0, B - 1):
        kv = [N if b == long_one else short for b in range(B)]
        run_attention(ctx, dtype, 64, B, 1, group, n_q, N, N + 1, kv, [min(n_q, max(1, n)) for n in kv], seed=N)


@pytest.mark.parametrize("d", [32, 256])
def test_row_blocks_and_key_blocks_in_pairs(ctx, d):
    """Calls large enough for workgroups to take two blocks each, an odd number of them."""
    run_attention(ctx, "f16", d, 8, 64, 1, 300, 513, 514, [513, 300, 1, 0, 257, 512, 400, 299], [300, 300, 1, 300, 0, 129, 300, 299])
