"""pctree_paged_attention against the float64 oracle.

Tolerance per output element, with A = sum_s p_s |v_s| and u the half step of
the type: probabilities rounded for the product u * A; scores, float32 sums of
D <= 128 products (at most 128 * 2^-24 of sum |q k| * scale, below 25 here:
2e-4) and the exponential change a probability by 2.5e-4 relative, numerator
and sum alike: 5e-4 * A; the output's rounding u * |out|.  In float16 a
probability below 2^-14 of its row's reference is rounded to 2^-25: keys *
2^-25 * max |v| more.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.kv_util import DTYPES, Batch, f64, half_step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


class Call:
    def __init__(self, P, b, Hq, Hkv, D, dtype="bf16", seed=0, q_pad=0, garbage=True):
        self.b, self.dt = b, DTYPES[dtype]
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        rnd = lambda *s: torch.randn(*s, generator=g, dtype=self.dt, device="cuda")
        wide = rnd(b.total, Hq * D + q_pad) * 1.5
        self.q = wide[:, :Hq * D].unflatten(1, (Hq, D))
        self.cfg = P.paged_attn_config(b.batch, b.total, Hq, Hkv, D, b.page_size, b.n_pages,
                                       b.max_pages, self.dt, q_stride=wide.stride(0))
        places = b.n_pages * b.page_size
        self.k, self.v = rnd(places, Hkv, D), rnd(places, Hkv, D)
        if garbage:                    # what no row sees holds anything
            free = np.ones(places, bool)
            for r in range(b.batch):
                free[b.places(r, 0, int(b.prefix[r] + b.rows[r]))] = False
            at = torch.from_numpy(np.flatnonzero(free)).cuda()
            self.k[at] = float("nan")
            self.v[at] = float("inf")
        self.out = torch.full((b.total + 2, Hq, D), 9.0, dtype=self.dt, device="cuda")
        nb = P.pctree_paged_attention_workspace_bytes(self.cfg)
        self.ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dev = b.dev()

    def args(self):
        return dict(q=self.q, k_cache=self.k, v_cache=self.v, out=self.out[1:-1],
                    workspace=self.ws, status=self.status, **self.dev)

    def run(self, P, **kw):
        P.pctree_paged_attention(self.cfg, **{**self.args(), **kw})
        torch.cuda.synchronize()
        return int(self.status.item())

    def want(self):
        b = self.b
        k, v = f64(self.k), f64(self.v)
        return O.paged_attention(f64(self.q), k, v, b.start, b.rows, b.prefix, b.page_size,
                                 b.table, self.cfg.scale)

    def check(self, want=None, rows=None):
        b, u = self.b, half_step(self.dt)
        out, size = self.want() if want is None else want
        got = f64(self.out)
        used = b.used_rows()
        assert (got[[0, -1]] == 9).all() and (got[1:-1][~used] == 9).all()
        tol = (u + 5e-4) * size + u * np.abs(out)
        if self.dt is torch.float16:
            tol += float(max(b.prefix + b.rows)) * 2.0 ** -25 * 6
        at = np.flatnonzero(used) if rows is None else rows
        err = np.abs(got[1:-1][at] - out[at])
        assert (err <= tol[at]).all(), (err - tol[at]).max()


SHAPES = {
    "one_key": dict(rows=[1], prefix=[0], page=16, heads=(32, 8)),
    "token": dict(rows=[1], prefix=[2047], page=16, heads=(32, 8)),
    "tokens": dict(rows=[1, 1, 1, 1, 1], prefix=[0, 127, 128, 700, 3], page=32, heads=(40, 8)),
    "tokens_contiguous": dict(rows=[1, 1, 1], prefix=[5, 300, 129], page=0, heads=(16, 16)),
    "chains": dict(rows=[8, 8, 3, 0, 8], prefix=[100, 250, 0, 9, 121], page=0, heads=(32, 8)),
    "prompt": dict(rows=[300], prefix=[0], page=16, heads=(10, 2)),
    "prompts_gaps": dict(rows=[129, 1, 64, 0, 200], prefix=[0, 40, 65, 3, 128], page=64,
                         heads=(8, 2), gap=2),
    "page_8": dict(rows=[40, 17], prefix=[90, 3], page=8, heads=(4, 2)),
    "page_1": dict(rows=[12, 3], prefix=[20, 0], page=1, heads=(4, 2)),
    "page_23": dict(rows=[40, 17], prefix=[90, 3], page=23, heads=(4, 2)),
    "page_100": dict(rows=[150, 17], prefix=[90, 203], page=100, heads=(4, 2)),
    "page_128": dict(rows=[150, 17], prefix=[90, 203], page=128, heads=(4, 2)),
    "page_200": dict(rows=[150, 17], prefix=[90, 403], page=200, heads=(4, 2)),
    "one_head": dict(rows=[140, 2], prefix=[7, 260], page=16, heads=(3, 3)),
    "wide_group": dict(rows=[5, 1], prefix=[130, 0], page=16, heads=(128, 1)),
    "group_of_48": dict(rows=[5, 9], prefix=[130, 0], page=32, heads=(96, 2)),
    # several tiles a request: pairs of CTAs, an odd tile, a last tile of one row
    "pairs_odd_tiles": dict(rows=[161, 33, 0, 70], prefix=[0, 300, 5, 77], page=16, heads=(16, 4)),
    "pairs_long_prefix": dict(rows=[65, 129], prefix=[1900, 3], page=64, heads=(16, 4), gap=1),
    "pairs_one_head": dict(rows=[500], prefix=[130], page=32, heads=(2, 2)),
    "pairs_wide_group": dict(rows=[9, 4], prefix=[250, 0], page=16, heads=(96, 2)),
    "many_requests": dict(rows=[1, 2, 1] * 40, prefix=[3, 0, 129] * 40, page=16, heads=(4, 4)),
}


for _page in (0, 1, 8, 16, 23, 32, 48, 64, 100, 128, 200):
    SHAPES[f"pairs_page_{_page}"] = dict(rows=[70, 41], prefix=[190, 3], page=_page, heads=(16, 2))

# clusters of four: many tiles a request, small pages
for _page in (1, 5, 8, 16):
    SHAPES[f"fours_page_{_page}"] = dict(rows=[205, 97, 0, 129], prefix=[40, 301, 7, 0],
                                         page=_page, heads=(16, 2), gap=1)


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "bf16"), (128, "f16"), (64, "f16")])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_shapes(P, name, D, dtype):
    s = SHAPES[name]
    b = Batch(s["rows"], s["prefix"], s["page"], gap=s.get("gap", 0))
    c = Call(P, b, *s["heads"], D, dtype, q_pad=8 if D == 64 else 0)
    assert c.run(P) == 0
    c.check()


def test_long_prefix_split_over_every_sm(P):
    b = Batch([1, 3], [20000, 9001], 64)
    c = Call(P, b, 8, 2, 128)
    assert c.run(P) == 0
    c.check()


def test_same_result_whatever_the_workspace_held(P):
    b = Batch([30, 1, 7], [500, 1000, 3], 16)
    c = Call(P, b, 16, 4, 128)
    assert c.run(P) == 0
    first = c.out.clone()
    c.ws.zero_()
    assert c.run(P) == 0
    assert torch.equal(first, c.out)


def test_peaked_and_growing_scores(P):
    """Maxima that grow along the keys move every row's reference, and scores
    far apart leave one key."""
    b = Batch([20, 1], [400, 300], 16)
    for factor in (0.02, 12.0):
        c = Call(P, b, 4, 2, 128, garbage=False)
        ramp = torch.arange(c.k.shape[0], device="cuda") / c.k.shape[0]
        c.q.mul_(0).add_(factor)
        c.k.copy_((ramp[:, None, None] * torch.ones_like(c.k).float()).to(c.dt))
        assert c.run(P) == 0
        out, size = c.want()
        got, u = f64(c.out[1:-1]), half_step(c.dt)
        # scores of up to 136 after the float32 sum of 128 equal terms: 1e-5 of
        # them absolute
        tol = (u + 2 * 1e-5 * 136 + 5e-4) * size + u * np.abs(out)
        assert (np.abs(got - out) <= tol).all()


def test_non_finite_keys_reach_only_the_rows_that_see_them(P):
    b = Batch([24, 5], [200, 30], 16)
    for value in (float("nan"), float("inf")):
        c = Call(P, b, 8, 2, 128)
        clean = c.want()
        slot = 200 + 10                              # row 10's own key, KV head 1
        at = int(b.places(0, slot, slot + 1)[0])
        c.k[at, 1, 5] = value
        with np.errstate(invalid="ignore"):
            want, size = c.want()
        assert c.run(P) == 0
        got = f64(c.out[1:-1])
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        assert np.isnan(want[10:24, 4:]).any() and not np.isnan(want[:10]).any()
        fin = ~np.isnan(want)
        u = half_step(c.dt)
        tol = (u + 5e-4) * size + u * np.abs(want)
        assert (np.abs(got - want)[fin] <= tol[fin]).all()
        del clean


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("page", [0, 8, 16, 100])
@pytest.mark.parametrize("rows,prefix", [([24, 5], [200, 30]), ([150, 90, 1], [0, 130, 40])])
def test_non_finite_values_reach_only_the_rows_that_see_them(P, rows, prefix, page, D, dtype):
    """Values of new rows' slots, seen by the later rows of their tile alone, and
    of prefix slots, seen by all."""
    b = Batch(rows, prefix, page)
    inf, nan = float("inf"), float("nan")
    c = Call(P, b, 8, 2, D, dtype)
    # (request, slot past the prefix, KV head, dim, value); row 0's own slot is
    # seen by every row, a pair of opposite infinities is NaN where both are seen
    places = [(0, 5, 1, 3, inf), (0, 9, 1, 3, -inf), (0, 12, 0, D - 1, nan), (0, 23, 1, 17, -inf),
              (1, 0, 0, 40, inf), (1, 4, 1, 0, nan), (0, rows[0] - 1, 0, 8, inf)]
    if prefix[1] > 3:
        places.append((1, -3, 1, 63, inf))
    for r, j, h, d, x in places:
        at = int(b.places(r, prefix[r] + j, prefix[r] + j + 1)[0])
        c.v[at, h, d] = x
    assert c.run(P) == 0
    # the reference without 0 * inf: finite values, then what each row sees
    k, v = f64(c.k), f64(c.v)
    finite = np.where(np.isfinite(v), v, 0.0)
    want, size = O.paged_attention(f64(c.q), k, finite, b.start, b.rows, b.prefix, b.page_size,
                                   b.table, c.cfg.scale)
    special = np.zeros(want.shape)
    with np.errstate(invalid="ignore"):
        for r, j, h, d, x in places:
            first = int(b.start[r]) + max(j, 0)
            special[first:int(b.start[r]) + rows[r], 4 * h:4 * h + 4, d] += x
        want = want + special
    got = f64(c.out[1:-1])
    used = b.used_rows()
    np.testing.assert_array_equal(np.isnan(got[used]), np.isnan(want[used]))
    np.testing.assert_array_equal(np.isinf(got[used]), np.isinf(want[used]))
    np.testing.assert_array_equal(np.sign(got[used][np.isinf(want[used])]),
                                  np.sign(want[used][np.isinf(want[used])]))
    fin = used[:, None, None] & np.isfinite(want)
    u = half_step(c.dt)
    tol = (u + 5e-4) * size + u * np.abs(np.where(fin, want, 0))
    if dtype == "f16":
        tol += float(max(b.prefix + b.rows)) * 2.0 ** -25 * 6
    assert (np.abs(np.where(fin, got - want, 0)) <= tol).all()


def test_many_non_finite_values(P):
    """More of them in a tile than are told apart: rows from the first on are
    NaN, those before it untouched."""
    b = Batch([32], [64], 16)
    c = Call(P, b, 8, 2, 128)
    clean = c.want()
    at = torch.from_numpy(b.places(0, 64 + 10, 64 + 32)).cuda()
    c.v[at] = float("nan")
    assert c.run(P) == 0
    got = f64(c.out[1:-1])
    assert np.isnan(got[10:]).all()
    c.check(clean, rows=np.arange(10))


def test_bad_requests_and_pages(P):
    b = Batch([3, 40, 2, 5], [4, 60, 30, 7], 8)
    c = Call(P, b, 4, 2, 64)
    full = c.want()
    for name, value in (("prefix_len", -1), ("prefix_len", b.max_pages * 8 - 4),
                        ("n_rows", -1), ("n_rows", 6), ("row_start", -1),
                        ("row_start", b.total - 4)):
        c = Call(P, b, 4, 2, 64)
        c.dev[name][3] = value
        assert c.run(P) == -1, name
        keep = b.rows.copy()
        b.rows[3] = 0                                # its rows stay as they were
        c.check(full)
        b.rows[:] = keep
    # a page number that is no page: zeros, no fault, other requests untouched
    c = Call(P, b, 4, 2, 64)
    c.dev["page_table"][1, 2] = b.n_pages + 5
    c.dev["page_table"][1, 3] = -1
    assert c.run(P) == -1
    got = f64(c.out[1:-1])
    assert np.isfinite(got[b.used_rows()]).all()
    c.check(full, rows=np.r_[0:3, 43:50])


def test_no_rows_at_all(P):
    b = Batch([0, 0], [4, 0], 16, gap=1)
    c = Call(P, b, 4, 2, 64)
    assert c.run(P) == 0
    assert (c.out == 9).all()


@pytest.mark.parametrize("page", [0, 16])
def test_as_many_requests_as_there_may_be(P, page):
    """1024 requests: none, one and several tiles of rows in any order."""
    rng = np.random.default_rng(3)
    rows = rng.choice([0, 1, 1, 1, 2, 5], 1024)
    rows[[0, 15, 16, 511, 512, 700, 1023]] = [70, 0, 33, 129, 40, 1, 65]
    prefix = rng.integers(0, 40, 1024)
    prefix[[3, 600]] = [300, 129]
    c = Call(P, Batch(rows.tolist(), prefix.tolist(), page), 4, 1, 64)
    assert c.run(P) == 0
    c.check()


def test_requests_that_share_the_pages_of_a_prefix(P):
    b = Batch([1, 40, 3], [100, 130, 96], 16)
    b.table[1, :6] = b.table[0, :6]
    b.table[2, :6] = b.table[0, :6]
    c = Call(P, b, 8, 2, 128)
    assert c.run(P) == 0
    c.check()


def test_two_calls_at_once(P):
    """On two streams, each with a workspace of its own: single tokens beside
    prompts in pairs and in clusters of four."""
    calls = [Call(P, Batch([1] * 20, [int(x) for x in range(5, 1005, 50)], 64), 16, 4, 128),
             Call(P, Batch([205, 300], [40, 7], 16, seed=1), 16, 2, 128, seed=1),
             Call(P, Batch([300, 90], [0, 333], 64, seed=2), 16, 2, 64, "f16", seed=2)]
    want = [c.want() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(calls, streams):
            P.pctree_paged_attention(c.cfg, **c.args(), stream=s)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert int(c.status.item()) == 0
        c.check(w)


def test_streams_and_graphs(P):
    """On another stream, and replayed from two graphs that share a workspace
    one after the other."""
    b = Batch([70, 1, 9], [5, 900, 20], 16)
    c = Call(P, b, 8, 2, 128)
    want = c.want()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.pctree_paged_attention(c.cfg, **c.args(), stream=s)
    torch.cuda.synchronize()
    c.check(want)
    d = Call(P, b, 8, 2, 128, seed=5)
    d.ws = c.ws
    graphs = []
    for x in (c, d):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            P.pctree_paged_attention(x.cfg, **x.args())
        graphs.append(g)
    for _ in range(3):
        c.out.fill_(9)
        d.out.fill_(9)
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    c.check(want)
    d.check()


def test_pages_past_32_bits(P):
    """Keys in the last pages of a cache of more than 2^32 elements."""
    Hkv, D, page = 64, 128, 64
    pages = (1 << 32) // (Hkv * D * page) + 4
    kc = torch.zeros(pages, page, Hkv, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32)
    n = 3 * page - 7
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.bfloat16, device="cuda")
    k, v = rnd(3 * page, Hkv, D), rnd(3 * page, Hkv, D)
    for i, p in enumerate(table[0].tolist()):
        kc[p], vc[p] = k[i * page:(i + 1) * page], v[i * page:(i + 1) * page]
    q = rnd(1, Hkv, D)
    i32 = dict(dtype=torch.int32, device="cuda")
    cfg = P.paged_attn_config(1, 1, Hkv, Hkv, D, page, pages, 3)
    ws = torch.empty(P.pctree_paged_attention_workspace_bytes(cfg), dtype=torch.uint8,
                     device="cuda")
    out = torch.empty_like(q)
    P.pctree_paged_attention(cfg, q, kc, vc, torch.zeros(1, **i32), torch.ones(1, **i32),
                             torch.full((1,), n - 1, **i32), out, ws, page_table=table.cuda())
    s = torch.einsum("hd,shd->hs", q[0].double(), k[:n].double()) * D ** -0.5
    p = s.softmax(-1)
    want = torch.einsum("hs,shd->hd", p, v[:n].double())
    size = torch.einsum("hs,shd->hd", p, v[:n].double().abs())
    u = half_step(torch.bfloat16)
    assert bool(((out[0].double() - want).abs() <= (u + 5e-4) * size + u * want.abs()).all())
