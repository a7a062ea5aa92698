"""pctree_kv8_compact at the end of a request's slots: codes and scales are the
oracle's."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv8_compact import Call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


def test_long_paths_of_no_tree_are_left_untouched(P):
    """Longer than a request's slots, with neighbours that ascend."""
    c = Call(P, 6, [5, 9, 2], 8, 2, 64, 4, 1, 60, 1, lens=[2, 2, 2])
    assert c.b.max_pages * c.b.page_size < 60
    w = c.want(skip=(2,))
    c.len[2] = 60
    c.idx[2] = np.resize([0, 1, 2, 3, 4, 5], 61)
    assert c.run(P) == -1
    c.check(w)
