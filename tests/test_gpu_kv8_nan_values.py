"""pctree_kv8_attention with many NaN codes in new rows' values: each reaches its own
dim of the rows that see it, and nothing else.  Tolerances as in
test_gpu_kv8_attention.py."""
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


def with_nan(c, Hkv, D, share, rows=None, seed=0):
    """Value codes of new rows become NaN, each with the probability `share`."""
    rng = np.random.default_rng(seed)
    v = c.vp.cache.view(torch.uint8).view(-1, Hkv, D)
    for r in range(c.b.batch):
        T, n = int(c.b.prefix[r]), int(c.b.rows[r])
        at = torch.from_numpy(c.b.places(r, T, T + n)).cuda()
        nan = rng.random((n, Hkv, D)) < share
        if rows is not None:
            nan[np.setdiff1d(np.arange(n), rows)] = False
        code = np.where(rng.random((n, Hkv, D)) < 0.5, 0x7f, 0xff).astype(np.uint8)
        v[at] = torch.where(torch.from_numpy(nan).cuda(), torch.from_numpy(code).cuda(), v[at])


FORMS = {"causal": None, "tree": dict(), "forest": dict(chain=0.0, roots=5),
         "siblings": dict(chain=0.0, roots=1)}


@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("share", [0.002, 0.05, 1.0])
@pytest.mark.parametrize("D,heads,page,block", [(128, (2, 1), 16, 1), (64, (12, 3), 23, 8),
                                                (128, (48, 1), 0, 128)])
def test_every_dim_of_every_row(P, form, share, D, heads, page, block):
    b = Batch([64, 1, 200], [100, 7, 33], page)
    kind = FORMS[form]
    c = Call(P, b, *heads, D, block, parent=None if kind is None else parents(b, **kind))
    with_nan(c, heads[1], D, share)
    assert c.run(P) == 0
    c.check()
    first = c.out.clone()
    for _ in range(5):
        c.out.fill_(9.0)
        assert c.run(P) == 0
        assert torch.equal(c.out.nan_to_num(7.0), first.nan_to_num(7.0))


def test_siblings_of_rows_without_numbers(P):
    """Nine rows of NaN values under one root: their siblings are numbers."""
    b = Batch([256], [130], 48)
    c = Call(P, b, 6, 3, 128, 1, parent=np.full(256, 0, np.int32))
    c.parent[0] = -1
    c.parent[200:] = np.arange(200, 256) - 100
    with_nan(c, 3, 128, 1.0, rows=np.arange(100, 109))
    assert c.run(P) == 0
    nan = c.out[1:-1].isnan().cpu().numpy()
    rows = np.flatnonzero(nan.any((1, 2))).tolist()
    assert rows == [*range(100, 109), *range(200, 209)] and nan[rows].all()
    c.check()
