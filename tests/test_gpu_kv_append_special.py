"""pctree_kv_append: frequencies that are not finite."""
import pytest
import torch

from tests.kv_util import Batch
from tests.test_gpu_kv_append import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("interleaved", [False, True])
def test_frequencies_that_are_not_finite(value, interleaved):
    """An error, and no angle for that pair; the others are turned."""
    from paper_2608_02123_gb300 import pctree as P
    c = Call(P, Batch([3, 2], [5, 0], 16), 4, 2, 128, interleaved=interleaved)
    c.freq[[0, 17, 63]] = value
    assert c.run(P) == -1
    c.freq[[0, 17, 63]] = 0.0
    c.check()
