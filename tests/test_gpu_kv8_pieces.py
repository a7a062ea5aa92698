"""pctree_kv8_attention where a CTA takes many short pieces.  Tolerances as in
test_gpu_kv8_attention.py."""
import pytest
import torch

from tests.kv_util import Batch
from tests.test_gpu_kv8_attention import Call, parents

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


# a group of 4 heads has 32 rows in a tile: requests of one tile, of two now and then
BATCHES = {
    "one_tile": ([3] * 250, [1, 70, 140, 5, 64] * 50),
    "one_tile_and_two": ([3, 1, 2, 40, 3, 3, 3, 3, 3, 3] * 25, [7, 0, 130, 64, 1] * 50),
    "two_tiles_first": ([60] + [2] * 200, [10] * 201),
}


@pytest.mark.parametrize("with_tree", [False, True])
@pytest.mark.parametrize("name", sorted(BATCHES))
def test_every_launch_gives_the_same(P, name, with_tree):
    """Warps of a unit's second tile have no part in units of one: however far they
    are behind, they find every later piece."""
    rows, prefix = BATCHES[name]
    b = Batch(rows, prefix, 16)
    c = Call(P, b, 32, 8, 64, 1)
    if with_tree:
        c.parent = parents(b)
    assert c.run(P) == 0
    c.check()
    first = c.out.clone()
    args = c.args()
    for _ in range(40):
        c.out.fill_(9.0)
        P.pctree_kv8_attention(c.cfg, **args)
        assert torch.equal(c.out, first)
    assert int(c.status.item()) == 0
