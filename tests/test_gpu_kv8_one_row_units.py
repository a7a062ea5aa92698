"""pctree_kv8_attention where rows are not more than requests, so that every row is a
unit of its own: trees and what is wrong with a call.  Tolerances as in
test_gpu_kv8_attention.py."""
import numpy as np
import pytest
import torch

from tests.kv_util import Batch, f64
from tests.test_gpu_kv8_attention import Call, parents

pytestmark = pytest.mark.gpu

# query and KV heads: groups of 4, 8, 9, 16 and 24
HEADS = [(8, 2), (8, 1), (18, 2), (32, 2), (24, 1)]


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


BATCHES = {
    "one_row_each": ([1, 1], [300, 0], 64),
    "siblings": ([4, 0, 0, 0], [33, 5, 0, 9], 16),
    "some_idle": ([3, 0, 1, 0, 2, 0], [70, 4, 0, 3, 515, 1], 16),
    "contiguous": ([9, 0, 0, 1] + [0] * 8, [20, 3, 1, 600] + [0] * 8, 0),
    "many_rows": ([70, 0, 3] + [0] * 70, [400, 3, 1] + [0] * 70, 23),
    "largest": ([256] + [0] * 255, [41] + [0] * 255, 48),
}


@pytest.mark.parametrize("D,dtype,block", [(128, "bf16", 1), (64, "f16", 8)])
@pytest.mark.parametrize("kind", [dict(chain=0.0, roots=3), dict(), dict(chain=1.0)])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("name", sorted(BATCHES))
def test_trees(P, name, heads, kind, D, dtype, block):
    rows, prefix, page = BATCHES[name]
    b = Batch(rows, prefix, page)
    assert b.total <= b.batch
    c = Call(P, b, *heads, D, block, dtype, parent=parents(b, **kind))
    assert c.run(P) == 0
    c.check()


@pytest.mark.parametrize("heads", [(8, 2), (18, 2), (24, 1)])
def test_nan_codes_of_unseen_rows_stay_there(P, heads):
    b = Batch([6, 0, 0, 0, 1, 0, 0], [37, 0, 3, 1, 90, 2, 2], 16)
    parent = np.array([-1, 0, 0, 1, 2, -1, -1], np.int32)
    c = Call(P, b, *heads, 128, 1, parent=parent)
    at = b.places(0, 37, 43)
    for p, row, dims in ((c.kp, 1, slice(5, 6)), (c.vp, 2, slice(60, 70)),
                         (c.vp, 5, slice(0, 128))):
        p.cache.view(torch.uint8).view(-1, heads[1], 128)[int(at[row]), :, dims] = 0x7f
    assert c.run(P) == 0
    got = f64(c.out)[1:-1]
    seen = np.isnan(got).any((1, 2))
    assert seen.tolist() == [False, True, True, True, True, True, False]
    c.check()


@pytest.mark.parametrize("heads", [(8, 2), (18, 2), (24, 1)])
def test_bad_parents(P, heads):
    b = Batch([1, 5, 0, 0, 0, 1, 0], [20, 40, 1, 2, 3, 0, 5], 16)
    good = np.array([-1, -1, 0, 0, -1, 2, -1], np.int32)
    c = Call(P, b, *heads, 64, parent=good.copy())
    assert c.run(P) == 0
    want = c.want()
    c.check(want)
    for row, bad in ((0, 0), (0, -2), (4, 3), (4, 300), (6, 2 ** 31 - 1), (1, -2 ** 31)):
        c.parent = good.copy()
        c.parent[row] = bad                    # counts as a root
        c.status.zero_()
        c.out.fill_(9.0)
        assert c.run(P) == -1
        c.check(want)


@pytest.mark.parametrize("heads", [(8, 2), (18, 2), (24, 1)])
def test_a_request_of_more_rows_than_a_tree_may_have(P, heads):
    b = Batch([257, 1] + [0] * 256, [3, 20] + [0] * 256, 16)
    c = Call(P, b, *heads, 64, parent=np.full(b.total, -1, np.int32))
    assert c.run(P) == -1
    got = f64(c.out)[1:-1]
    assert (got[:257] == 9).all() and (got[257] != 9).any()
    c.check(rows=[257])


@pytest.mark.parametrize("heads", [(8, 2), (18, 2), (24, 1)])
def test_bad_scales_pages_and_requests(P, heads):
    b = Batch([1] * 6, [100, 40, 50, 30, 0, 700], 16)
    c = Call(P, b, *heads, 128, 1)
    for r, key, byte in ((0, 7, 255), (5, 640, 0)):
        c.vp.scale.view(torch.uint8).view(-1, heads[1])[int(b.places(r, key, key + 1)[0]), 0] = byte
    c.kp.scale.view(torch.uint8).view(-1, heads[1])[int(b.places(3, 2, 3)[0]), 0] = 3
    assert c.run(P) == -1
    for p in (c.vp, c.kp):                               # what they count as
        scales = p.scale.view(torch.uint8)
        scales.copy_(scales.clamp(127 - 15, 127 + 7))
    want = c.want()
    c.check(want)
    c.status.zero_()
    assert c.run(P) == 0
    c.check(want)
    for name, r, value in (("n_rows", 2, -1), ("prefix_len", 3, b.max_pages * b.page_size),
                           ("row_start", 4, 6)):
        c.dev = b.dev()
        c.dev[name][r] = value
        c.status.zero_()
        c.out.fill_(9.0)
        assert c.run(P) == -1
        assert (f64(c.out)[1 + r] == 9).all()
        c.check(want, rows=[x for x in range(6) if x != r])


@pytest.mark.parametrize("number", [-3, 1 << 30])
@pytest.mark.parametrize("heads", [(8, 2), (18, 2), (24, 1)])
def test_a_bad_page_is_a_page_of_zeros(P, heads, number):
    b = Batch([1] * 3, [100, 40, 7], 16)
    c = Call(P, b, *heads, 128, 4)
    free = int(np.setdiff1d(np.arange(b.n_pages), b.table)[0])
    for p in (c.kp, c.vp):
        p.cache.view(torch.uint8)[free] = 0
    right = int(b.table[0, 2])
    c.dev["page_table"][0, 2] = number
    assert c.run(P) == -1
    b.table[0, 2] = free
    c.check()
    b.table[0, 2] = right
