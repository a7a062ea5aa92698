"""pctree_paged_attention where scores or values are not finite in more than one
way at a time: what the formula gives in float64, NaN and infinities included.

Tolerances of the finite elements are those of test_gpu_paged_attention.py.
"""
import numpy as np
import pytest
import torch

from tests.kv_util import Batch, f64, half_step
from tests.test_gpu_paged_attention import Call

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


def put(c, cache, r, slot, head, dim, value):
    at = int(c.b.places(r, slot, slot + 1)[0])
    cache[at, head, dim] = value


def compare(c):
    b = c.b
    with np.errstate(invalid="ignore"):
        want, size = c.want()
    used = b.used_rows()
    got, want, size = f64(c.out[1:-1])[used], want[used], size[used]
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(np.isposinf(got), np.isposinf(want))
    np.testing.assert_array_equal(np.isneginf(got), np.isneginf(want))
    fin = np.isfinite(want)
    u = half_step(c.dt)
    tol = (u + 5e-4) * size[fin] + u * np.abs(want[fin])
    if c.dt is torch.float16:
        tol += float(max(b.prefix + b.rows)) * 2.0 ** -25 * 6
    assert (np.abs(got[fin] - want[fin]) <= tol).all()
    return want


# whole units, and units cut into pieces that are joined
PREFIXES = {"whole": [200, 30], "pieces": [9000, 2500]}


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("name", sorted(PREFIXES))
def test_infinite_values_of_new_rows_do_not_hide_what_came_before(P, name, D, dtype):
    """A new row's infinite value, in a row that is NaN already (a NaN score) or
    holds the opposite infinity (a value of the prefix)."""
    prefix = PREFIXES[name]
    c = Call(P, Batch([12, 5], prefix, 64), 8, 2, D, dtype)
    T = prefix[0]
    put(c, c.k, 0, T + 3, 0, 7, NAN)              # rows from 3 on of head 0: NaN
    put(c, c.v, 0, T + 5, 0, 11, INF)             # and from 5 on also an infinite value
    put(c, c.v, 0, T + 6, 0, 12, -INF)
    put(c, c.v, 0, 17, 1, 20, -INF)               # seen by every row of head 1
    put(c, c.v, 0, T + 4, 1, 20, INF)             # opposite: NaN from row 4 on
    put(c, c.v, 0, 18, 1, 33, INF)
    put(c, c.v, 0, T + 4, 1, 33, INF)             # the same sign: stays infinite
    assert c.run(P) == 0
    want = compare(c)
    assert np.isnan(want[5:12, :4, 11]).all() and np.isnan(want[4:12, 4:, 20]).all()
    assert np.isneginf(want[:4, 4:, 20]).all() and np.isposinf(want[:12, 4:, 33]).all()


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "f16")])
def test_rows_whose_scores_are_all_minus_infinity(P, D, dtype):
    """Such a row has no softmax: NaN.  With one finite score among them it is
    that key's value."""
    c = Call(P, Batch([1, 3, 1, 2], [0, 0, 9000, 130], 64), 8, 2, D, dtype)
    c.q[..., 5] = 1.0
    b = c.b

    def sink(r, first, last):
        at = torch.from_numpy(b.places(r, first, last)).cuda()
        c.k[at, :, 5] = -INF

    sink(0, 0, 1)                                 # the only key
    sink(1, 0, 1)                                 # the first row's only key
    sink(2, 0, 9001)                              # every key, over many CTAs
    sink(3, 0, 130)                               # all but the rows' own
    assert c.run(P) == 0
    want = compare(c)
    assert np.isnan(want[[0, 1, 4]]).all() and np.isfinite(want[[2, 3, 5, 6]]).all()


def test_requests_that_claim_the_same_rows(P):
    """More rows together than there are: an error, and nothing is written."""
    c = Call(P, Batch([30, 7, 1], [100, 20, 0], 16), 4, 2, 64)
    c.dev["row_start"].zero_()
    c.dev["n_rows"].copy_(torch.tensor([38, 7, 1]))
    c.dev["prefix_len"].copy_(torch.tensor([80, 20, 0]))
    assert c.run(P) == -1
    assert (c.out == 9).all()
    b = Batch([30, 7, 1], [100, 20, 0], 16)          # and as many as there are
    c = Call(P, b, 4, 2, 64)
    assert c.run(P) == 0
    c.check()


@pytest.mark.parametrize("D,dtype,power", [(64, "bf16", 30), (64, "bf16", 58), (128, "bf16", 40),
                                           (64, "f16", 27), (128, "f16", 27)])
@pytest.mark.parametrize("name", sorted(PREFIXES))
def test_scores_too_large_for_fractions(P, name, D, dtype, power):
    """Scores whose floats are whole numbers apart (2^power and more): the largest
    takes all, exactly."""
    prefix = PREFIXES[name]
    b = Batch([12, 5], prefix, 64)
    c = Call(P, b, 8, 2, D, dtype, garbage=False)
    # one product a score, four times or D times the same: exact in float32
    n = 4 if dtype == "bf16" else D
    c.q.zero_()
    c.k.zero_()
    half = power // 2
    g = torch.Generator(device="cuda")
    g.manual_seed(power)
    steps = torch.randint(-128, 128, c.k.shape[:2], generator=g, device="cuda")
    if half > 14:                                # float16 ends at 2^16
        c.q[..., :n] = 2.0 ** (power - half)
        c.k[..., :n] = ((1 + steps / 128.0) * 2.0 ** half)[..., None].to(c.dt)
    else:
        c.q[..., :n] = 2.0 ** 14
        c.k[..., :n] = ((1 + steps / 128.0) * 2.0 ** (power - 14))[..., None].to(c.dt)
    # a largest one early in the prefix, one among the new rows
    for r in range(2):
        at = int(b.places(r, 9, 10)[0])
        c.k[at, :, :n] = 2.25 * 2.0 ** (half if half > 14 else power - 14)
        at = int(b.places(r, prefix[r] + 3, prefix[r] + 4)[0])
        c.k[at, :, :n] = 2.5 * 2.0 ** (half if half > 14 else power - 14)
    assert c.run(P) == 0
    got, v = c.out[1:-1], c.v
    for r in range(2):
        for j in range(int(b.rows[r])):
            at = int(b.places(r, 9, 10)[0] if j < 3 else b.places(r, prefix[r] + 3,
                                                                  prefix[r] + 4)[0])
            want = v[at].repeat_interleave(4, 0)
            assert torch.equal(got[int(b.start[r]) + j], want), (r, j)
