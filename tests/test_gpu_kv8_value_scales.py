"""pctree_kv8_attention where one key's values have a much larger scale than the
others', in dims of its own: what the others hold in theirs is not lost.

Tolerance per output dim, as in test_gpu_kv8_attention.py with what float16 has for
a probability p of a row's largest 1: 2^-11 of p, or 2^-25 where that is more.  With
A = sum_s p_s |v_s| (p normed) that is 2^-11 * A + 2^-25 * sum_s |v_s| (the norm's sum
is 1 at least), scores 5e-4 * A, the output's rounding u * |out| + 2^-25.
"""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from tests.kv_util import Batch, f64, half_step
from tests.test_gpu_kv8_attention import Call, parents

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


def check_dims(c):
    """Every dim for itself."""
    b, u = c.b, half_step(c.dt)
    out, size = c.want()
    got = f64(c.out)[1:-1]
    V = np.abs(c.values()[1])
    G = got.shape[1] // V.shape[1]
    for r in range(b.batch):
        at = b.places(r, 0, int(b.prefix[r] + b.rows[r]))
        total = V[at].sum(0).repeat(G, axis=0)                    # [Hq][D]
        rows = np.arange(b.start[r], b.start[r] + b.rows[r])
        tol = (2.0 ** -11 + 5e-4) * size[rows] + 2.0 ** -25 * total + u * np.abs(out[rows]) \
            + 2.0 ** -25
        err = np.abs(got[rows] - out[rows])
        assert (err <= tol).all(), (r, (err / tol).max())


@pytest.mark.parametrize("rows,with_tree", [([1], False), ([1, 1, 1], False), ([30], False),
                                            ([30], True), ([3, 0, 0], True)])
@pytest.mark.parametrize("D,dtype,heads", [(128, "bf16", (5, 1)), (64, "f16", (4, 2)),
                                           (128, "f16", (12, 1))])
@pytest.mark.parametrize("small,large", [(-15, 7), (-9, 7), (-8, 7), (-5, -2), (-5, -1)])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_one_large_scale(P, rows, with_tree, D, dtype, heads, small, large, where):
    T = 4000
    b = Batch(rows, [T] * len(rows), 64)
    Hq, Hkv = heads
    c = Call(P, b, Hq, Hkv, D, 1, dtype, garbage=False, parent=parents(b) if with_tree else None)
    c.q.zero_()
    c.q[:, :, 0] = 8.0
    k, v = (p.cache.view(torch.uint8).view(-1, Hkv, D) for p in (c.kp, c.vp))
    k.zero_()
    c.kp.scale.view(torch.uint8).fill_(O8.BIAS)
    c.vp.scale.view(torch.uint8).fill_(O8.BIAS + small)
    vs = c.vp.scale.view(torch.uint8).view(-1, Hkv)
    for r in range(b.batch):
        n = int(b.rows[r])
        p = int(b.places(r, 0, T)[{"first": 0, "middle": T // 2, "last": T - 1}[where]])
        # 8 * 10 / sqrt(128) in log2 units: its weight is 2^10 times another's at least
        k[p, :, 0] = int(O8.encode(10.0))
        vs[p] = O8.BIAS + large
        v[p] = 0
        v[p, :, 0] = int(O8.encode(448.0))
        v[p, :, 1] = int(O8.encode(-2.0 ** -9))
    assert c.run(P) == 0
    check_dims(c)


@pytest.mark.parametrize("rows,heads", [([1] * 5, (8, 2)), ([1] * 5, (16, 1)), ([40, 3], (8, 2))])
@pytest.mark.parametrize("exps", [(-15, 7), (-8, -5), (-8, -4), (-15, -15), (7, 7)])
def test_scales_of_every_slot_at_random(P, rows, heads, exps):
    rng = np.random.default_rng(1)
    b = Batch(rows, [700, 40, 300, 5, 64][:len(rows)], 16)
    c = Call(P, b, *heads, 128, 1, garbage=False)
    e = rng.integers(exps[0], exps[1] + 1, c.vp.scale.numel()).astype(np.uint8) + O8.BIAS
    s = c.vp.scale.view(torch.uint8)
    s.copy_(torch.from_numpy(e.astype(np.uint8)).cuda().view(s.shape))
    # dims are a slot's own: a number in every eighth
    places = b.n_pages * b.page_size
    keep = (np.arange(128)[None] + np.arange(places)[:, None]) % 8 == 0
    v = c.vp.cache.view(torch.uint8).view(places, heads[1], 128)
    v.mul_(torch.from_numpy(keep.astype(np.uint8)).cuda()[:, None])
    assert c.run(P) == 0
    check_dims(c)
