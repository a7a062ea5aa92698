"""pctree_kv8_attention with queries and softmax scales at the ends of float32.
Tolerances as in test_gpu_kv8_attention.py."""
import numpy as np
import pytest
import torch

from tests.kv_util import Batch
from tests.test_gpu_kv8_attention import Call, parents

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


@pytest.mark.parametrize("rows,with_tree", [([1, 1], False), ([40, 3], False), ([40, 3], True)])
@pytest.mark.parametrize("scale", [1e-31, 1e-12, 1e-45])
def test_rows_of_zeros_under_a_small_scale(P, rows, with_tree, scale):
    """Their scores are all 0: the mean of the values that they see."""
    b = Batch(rows, [300, 7], 16)
    c = Call(P, b, 8, 2, 128, parent=parents(b) if with_tree else None,
             q_size=min(1.5 * 128 ** -0.5 / scale, 1e38))
    c.cfg.scale = scale
    c.q[:, ::2] = 0.0
    c.q[0, 1] *= 2.0 ** -120
    assert c.run(P) == 0
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [[1, 1], [40, 3]])
def test_keys_of_zeros_under_a_large_scale(P, rows, dtype):
    """One key with a product that is not 0, far below the zeros of all others."""
    b = Batch(rows, [300, 7], 16)
    c = Call(P, b, 8, 2, 128, dtype=dtype, garbage=False)
    places = b.n_pages * b.page_size
    c.cfg.scale = 2.0 ** 90
    c.q.zero_()
    c.q[:, :, 3] = 2.0 ** 126 if dtype == "bf16" else 2.0 ** 15
    k = c.kp.cache.view(torch.uint8).view(places, 2, 128)
    k.zero_()
    c.kp.scale.view(torch.uint8).fill_(127 + 7)
    for r in range(2):
        k[int(b.places(r, 5, 6)[0]), :, 3] = 0x81            # -2^-9
    assert c.run(P) == 0
    # (float64 holds the scores)
    c.check()
