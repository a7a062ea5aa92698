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


@pytest.mark.parametrize("block", [1, 8, 64])
@pytest.mark.parametrize("page", [0, 16, 23])
def test_trees_smaller_than_the_packed_size(P, page, block):
    """A tree of 8 nodes that fills its request's last slots, although trees of 40
    would not fit there."""
    c = Call(P, 8, [130, 3, 76, 0], page, 2, 64, block, 2, 5, 1, lens=[5, 4, 0, 5])
    c.idx[0, :6] = [0, 1, 3, 4, 6, 7]
    c.cfg.N = 40
    b = c.b
    assert 130 + 40 > b.max_pages * b.page_size >= 138
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


@pytest.mark.parametrize("past", [None, -1, 1, 2 ** 31 - 1])
@pytest.mark.parametrize("page", [0, 16])
def test_paths_past_the_last_slot_are_left_untouched(P, page, past):
    c = Call(P, 12, [40, 7], page, 2, 64, 4, 2, 11, 1, lens=[3, 3])
    c.idx[0, :4] = [0, 2, 5, 9]
    c.cfg.N = 40
    slots = c.b.max_pages * c.b.page_size
    w = c.want(skip=(0,))
    a = c.args()
    # node 9 one past the last slot; no prefix; all rows past the last slot
    a["prefix_len"][0] = slots - 9 if past is None else slots if past == 1 else past
    assert c.run(P, **a) == -1
    c.check(w)


def test_long_paths_of_no_tree_are_left_untouched(P):
    """Longer than a request's slots, with neighbours that ascend."""
    c = Call(P, 6, [5, 9, 2], 8, 2, 64, 4, 1, 60, 1, lens=[2, 2, 2])
    assert c.b.max_pages * c.b.page_size < 60
    w = c.want(skip=(2,))
    c.len[2] = 60
    c.idx[2] = np.resize([0, 1, 2, 3, 4, 5], 61)
    assert c.run(P) == -1
    c.check(w)
