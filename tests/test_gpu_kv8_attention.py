"""pctree_kv8_attention against the float64 oracle on the cache's values.

Tolerance per output element, with A = sum_s p_s |v_s| and u the half step of
the type: each probability is rounded for the product with the values, by at
most 2^-11 of itself, or 2^-32 where it is below 2^-21 of its row's reference:
2^-11 * A + keys * 2^-32 * max |v|; scores are float32 sums of D <= 128 products
(at most 128 * 2^-24 of sum |q k| * scale, below 25 here: 2e-4) and with the
exponential change a probability by 2.5e-4 relative, numerator and sum alike:
5e-4 * A; the output's rounding is u * |out| (2^-25 where float16 is
subnormal).
"""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from tests.kv8_util import Plane
from tests.kv_util import DTYPES, Batch, f64, half_step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


class Call:
    def __init__(self, P, b, Hq, Hkv, D, block=1, dtype="bf16", seed=0, q_pad=0, parent=None,
                 garbage=True, q_size=1.5, as_bytes=False):
        self.b, self.dt, self.block = b, DTYPES[dtype], block
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        wide = torch.randn(b.total, Hq * D + q_pad, generator=g, dtype=self.dt,
                           device="cuda") * q_size
        self.q = wide[:, :Hq * D].unflatten(1, (Hq, D))
        self.cfg = P.kv8_attn_config(b.batch, b.total, Hq, Hkv, D, b.page_size, b.n_pages,
                                     b.max_pages, block, self.dt, q_stride=wide.stride(0))
        self.kp = Plane(b, Hkv, D, block, seed + 1, as_bytes=as_bytes)
        self.vp = Plane(b, Hkv, D, block, seed + 2, as_bytes=as_bytes)
        if garbage:                    # what no row sees holds anything
            free = np.ones(b.n_pages * b.page_size, bool)
            for r in range(b.batch):
                free[b.places(r, 0, int(b.prefix[r] + b.rows[r]))] = False
            at = torch.from_numpy(np.flatnonzero(free)).cuda()
            for p in (self.kp, self.vp):
                p.cache.view(torch.uint8).view(-1, Hkv, D)[at] = 0x7f
        self.parent = parent
        self.out = torch.full((b.total + 2, Hq, D), 9.0, dtype=self.dt, device="cuda")
        nb = P.pctree_kv8_attention_workspace_bytes(self.cfg)
        self.ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dev = b.dev()

    def args(self):
        return dict(q=self.q, k_cache=self.kp.cache, v_cache=self.vp.cache,
                    k_scale=self.kp.scale, v_scale=self.vp.scale, out=self.out[1:-1],
                    workspace=self.ws, status=self.status,
                    parent=None if self.parent is None else
                    torch.from_numpy(self.parent).cuda(), **self.dev)

    def run(self, P, **kw):
        P.pctree_kv8_attention(self.cfg, **{**self.args(), **kw})
        torch.cuda.synchronize()
        return int(self.status.item())

    def values(self):
        return [O8.values(*(a[0] for a in p.bytes()), self.b.page_size, self.block)
                for p in (self.kp, self.vp)]

    def want(self):
        b = self.b
        return O8.attention(f64(self.q), *self.values(), b.start, b.rows, b.prefix, b.page_size,
                            b.table, self.cfg.scale, self.parent)

    def check(self, want=None, rows=None):
        b, u = self.b, half_step(self.dt)
        out, size = self.want() if want is None else want
        got = f64(self.out)
        used = b.used_rows()
        assert (got[[0, -1]] == 9).all() and (got[1:-1][~used] == 9).all()
        top = np.nanmax(np.abs(self.values()[1]))
        tol = (2.0 ** -11 + 5e-4) * size + u * np.abs(out) + 2.0 ** -25
        tol = tol + float(max(b.prefix + b.rows)) * 2.0 ** -32 * top
        at = np.flatnonzero(used) if rows is None else rows
        g, o = got[1:-1][at], out[at]
        assert (np.isnan(g) == np.isnan(o)).all()
        err = np.where(np.isnan(o), 0.0, np.abs(g - o))
        assert (err <= np.where(np.isnan(o), 0.0, tol[at])).all(), np.nanmax(err - tol[at])


def tree(n, seed=0, chain=0.3, roots=1):
    """Parents of a packed tree: parent[i] < i."""
    rng = np.random.default_rng(seed)
    p = [-1] * min(n, roots)
    for i in range(len(p), n):
        p.append(i - 1 if rng.random() < chain else int(rng.integers(0, i)))
    return p


def parents(b, **kw):
    out = np.full(b.total, -1, np.int32)
    for r, (a, n) in enumerate(zip(b.start, b.rows)):
        out[a:a + n] = tree(int(n), seed=r, **kw)
    return out


SHAPES = {
    "one_key": dict(rows=[1], prefix=[0], page=16, heads=(32, 8)),
    "token": dict(rows=[1], prefix=[2047], page=16, heads=(32, 8)),
    "tokens": dict(rows=[1, 1, 1, 1, 1], prefix=[0, 127, 128, 700, 3], page=32, heads=(40, 8)),
    # two groups of eight heads in the kernel for single tokens
    "tokens_group_of_9": dict(rows=[1, 1, 1], prefix=[5, 300, 1029], page=16, heads=(18, 2)),
    "tokens_group_of_16": dict(rows=[1] * 7, prefix=[0, 15, 16, 31, 32, 800, 2100], page=48,
                               heads=(32, 2)),
    "tokens_contiguous": dict(rows=[1, 1, 1], prefix=[5, 300, 129], page=0, heads=(16, 16)),
    "chains": dict(rows=[8, 8, 3, 0, 8], prefix=[100, 250, 0, 9, 121], page=0, heads=(32, 8)),
    "pairs": dict(rows=[2, 1, 2], prefix=[100, 250, 0], page=16, heads=(16, 4)),
    "prompt": dict(rows=[300], prefix=[0], page=16, heads=(10, 2)),
    "prompts_gaps": dict(rows=[129, 1, 64, 0, 200], prefix=[0, 40, 65, 3, 128], page=64,
                         heads=(8, 2), gap=2),
    "one_head": dict(rows=[140, 2], prefix=[7, 260], page=16, heads=(3, 3)),
    "wide_group": dict(rows=[5, 1], prefix=[130, 0], page=16, heads=(128, 1)),
    "group_of_48": dict(rows=[5, 9], prefix=[130, 0], page=32, heads=(96, 2)),
    "group_of_24": dict(rows=[1, 1], prefix=[130, 511], page=32, heads=(24, 1)),
    "long_prefix": dict(rows=[65, 129], prefix=[1900, 3], page=64, heads=(16, 4), gap=1),
    "many_requests": dict(rows=[1, 2, 1] * 40, prefix=[3, 0, 129] * 40, page=16, heads=(4, 4)),
    "many_tokens": dict(rows=[1] * 90, prefix=[3, 700, 129] * 30, page=16, heads=(8, 2)),
}
for _page in (0, 1, 8, 23, 64, 100, 128, 200):
    SHAPES[f"page_{_page}"] = dict(rows=[70, 41], prefix=[190, 3], page=_page, heads=(16, 2))


@pytest.mark.parametrize("D,dtype,block", [(128, "bf16", 1), (64, "bf16", 16), (128, "f16", 4),
                                           (64, "f16", 128)])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_shapes(P, name, D, dtype, block):
    s = SHAPES[name]
    b = Batch(s["rows"], s["prefix"], s["page"], gap=s.get("gap", 0))
    c = Call(P, b, *s["heads"], D, block, dtype, q_pad=8 if D == 64 else 0, as_bytes=D == 64)
    assert c.run(P) == 0
    c.check()


TREES = {
    "small": dict(rows=[9, 1, 16], prefix=[30, 0, 100], page=0, heads=(8, 2)),
    "wide": dict(rows=[64, 33, 0, 70], prefix=[1, 127, 9, 250], page=16, heads=(40, 8)),
    "largest": dict(rows=[256, 200], prefix=[129, 0], page=48, heads=(6, 3)),
    "one_group": dict(rows=[20], prefix=[300], page=64, heads=(32, 1)),
    "tokens": dict(rows=[1, 1], prefix=[300, 0], page=64, heads=(8, 2)),
}


@pytest.mark.parametrize("D,dtype,block", [(128, "bf16", 1), (64, "f16", 8)])
@pytest.mark.parametrize("kind", [dict(), dict(chain=1.0), dict(chain=0.0, roots=3)])
@pytest.mark.parametrize("name", sorted(TREES))
def test_trees(P, name, kind, D, dtype, block):
    s = TREES[name]
    b = Batch(s["rows"], s["prefix"], s["page"], gap=1)
    c = Call(P, b, *s["heads"], D, block, dtype, parent=parents(b, **kind))
    assert c.run(P) == 0
    c.check()


def test_a_chain_as_a_tree_is_causal(P):
    b = Batch([40, 8, 256], [77, 300, 1], 16)
    c = Call(P, b, 8, 2, 128)
    assert c.run(P) == 0
    causal = c.out.clone()
    c.parent = parents(b, chain=1.0)
    assert c.run(P) == 0
    assert torch.equal(c.out, causal)


def test_agrees_with_the_tree_attention_on_the_same_values(P):
    """Against pctree_tree_attention over the values in bfloat16 (exact there)."""
    N, prefix = 48, [200, 33]
    b = Batch([N, 20], prefix, 0)
    b.start = np.array([0, N], np.int32)
    b.total = 2 * N
    c = Call(P, b, 16, 4, 128, garbage=False)
    c.parent = np.full(2 * N, -1, np.int32)
    c.parent[:N], c.parent[N:N + 20] = tree(N, 5), tree(20, 6)
    assert c.run(P) == 0
    k, v = (torch.from_numpy(x).to(torch.bfloat16).cuda() for x in c.values())
    out = torch.zeros(2, N, 16, 128, dtype=torch.bfloat16, device="cuda")
    cfg = P.attn_config(2, N, 16, 4, b.page_size)
    nb = P.pctree_tree_attention_workspace_bytes(cfg)
    ws = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    P.pctree_tree_attention(cfg, c.q.contiguous(), k, v, c.dev["prefix_len"], c.dev["n_rows"],
                            torch.from_numpy(c.parent).cuda(), out, ws)
    torch.cuda.synchronize()
    want = f64(out.view(2 * N, 16, 128))
    used = b.used_rows()
    _, size = c.want()
    # each side's tolerance against the oracle
    tol = 2 * ((2.0 ** -8 + 5e-4) * size + 2.0 ** -8 * np.abs(np.nan_to_num(want)))
    assert (np.abs(f64(c.out)[1:-1] - want)[used] <= tol[used]).all()


def test_long_prefix_split_over_every_sm(P):
    b = Batch([1, 3], [20000, 9001], 64)
    c = Call(P, b, 8, 2, 128, 16)
    assert c.run(P) == 0
    c.check()


@pytest.mark.parametrize("rows", [[30, 1, 7], [1, 1, 1]])
def test_same_result_whatever_the_workspace_held(P, rows):
    b = Batch(rows, [500, 1000, 3], 16)
    c = Call(P, b, 16, 4, 128)
    assert c.run(P) == 0
    first = c.out.clone()
    c.ws.zero_()
    assert c.run(P) == 0
    assert torch.equal(first, c.out)


@pytest.mark.parametrize("rows,tree_rows", [([1], False), ([40], False), ([40], True)])
def test_a_far_tail_of_small_probabilities_is_kept(P, rows, tree_rows):
    """One key far above thousands of equal ones, which together weigh as much."""
    T = 6000
    b = Batch(rows, [T], 64)
    c = Call(P, b, 1, 1, 128, garbage=False)
    c.q.zero_()
    c.q[:, :, 0] = 8.0
    code = c.kp.cache.view(torch.uint8).view(-1, 1, 128)
    code.zero_()
    c.kp.scale.view(torch.uint8).fill_(127)
    p = b.places(0, 0, T + rows[0])
    # exp(8 * 12 / sqrt(128)) = 4842 times the others' weight
    code[int(p[5]), 0, 0] = int(O8.encode(12.0))
    if tree_rows:
        c.parent = parents(b)
    assert c.run(P) == 0
    c.check()


@pytest.mark.parametrize("rows", [[1, 1], [33, 20]])
def test_large_and_small_queries(P, rows):
    b = Batch(rows, [300, 7], 16)
    for size in (1e-30, 1e-6, 1e4, 1e30):
        c = Call(P, b, 8, 2, 128, q_size=size)
        # scores as at size 1.5
        c.cfg.scale = c.cfg.scale * 1.5 / size if size < 1e30 else 1e-31
        assert c.run(P) == 0
        c.check()


@pytest.mark.parametrize("rows", [[1], [6, 1], [70]])
def test_scales_of_all_sizes(P, rows):
    """Blocks whose scales are 2^-15 .. 2^7 times their codes."""
    b = Batch(rows, [400] * len(rows), 16)
    c = Call(P, b, 4, 2, 128, 2, garbage=False)
    c.vp = Plane(b, 2, 128, 2, 5, exps=(-15, 7))
    c.kp = Plane(b, 2, 128, 2, 6, exps=(-15, -7))
    assert c.run(P) == 0
    c.check()


@pytest.mark.parametrize("rows,prefix,with_tree", [
    ([1], [300], False), ([40], [300], False), ([8, 8], [40, 130], False), ([40], [300], True),
    ([1, 1, 1], [5, 600, 3], False), ([7], [0], True)])
def test_nan_codes_reach_the_rows_that_see_them(P, rows, prefix, with_tree):
    b = Batch(rows, prefix, 16)
    c = Call(P, b, 4, 2, 128, 1, parent=parents(b) if with_tree else None)
    k, v = (p.cache.view(torch.uint8).view(-1, 2, 128) for p in (c.kp, c.vp))
    for r, (n, T) in enumerate(zip(rows, prefix)):
        at = b.places(r, 0, T + n)
        if T > 0:
            v[int(at[T // 2]), 0, 77] = 0xff             # every row sees it
        v[int(at[T + n - 1]), 1, 3] = 0x7f               # the last row only
        v[int(at[T + n // 2]), 0, 100:103] = 0x7f
        k[int(at[T + n - 1]), 0, 5] = 0x7f
    assert c.run(P) == 0
    c.check()


def test_many_nan_values(P):
    b = Batch([64], [100], 16)
    c = Call(P, b, 2, 1, 128, 1)
    v = c.vp.cache.view(torch.uint8).view(-1, 1, 128)
    at = b.places(0, 100, 164)
    v[torch.from_numpy(at[20:60]).cuda()] = 0x7f
    assert c.run(P) == 0
    out, size = c.want()
    out[20:] = np.nan
    c.check((out, size))


def test_bad_scales_pages_and_requests(P):
    b = Batch([5, 1, 1, 4], [100, 40, 50, 30], 16)
    c = Call(P, b, 4, 2, 128, 1)
    c.vp.scale.view(torch.uint8).view(-1, 2)[int(b.places(0, 7, 8)[0]), 0] = 255
    assert c.run(P) == -1
    scales = c.vp.scale.view(torch.uint8)
    scales.copy_(scales.clamp(max=127 + 7))              # what it counts as
    c.check()
    c.status.zero_()
    c.dev["page_table"][1, 1] = -3                       # slots 16 .. 31: zeros
    c.dev["n_rows"][2] = -1
    c.dev["prefix_len"][3] = b.max_pages * b.page_size
    c.out.fill_(9.0)
    assert c.run(P) == -1
    got = f64(c.out)[1:-1]
    assert (got[6:] == 9).all() and np.isfinite(got[:6]).all() and (got[:6] != 9).any()


def test_bad_parents(P):
    b = Batch([10, 300], [20, 0], 16)
    c = Call(P, b, 4, 2, 128, parent=np.full(310, -1, np.int32))
    good = np.array([-1, 0, 1, 2, 1, 0, -1, 3, 4, 8], np.int32)
    c.parent[:10] = good
    assert c.run(P) == -1                                # 300 rows are no tree
    want = c.want()
    got = f64(c.out)[1:-1]
    assert (got[10:] == 9).all()
    first = c.out.clone()
    c.dev["n_rows"][1] = 0
    c.status.zero_()
    assert c.run(P) == 0
    assert torch.equal(first, c.out)
    c.parent[3], c.parent[5] = 7, -5                     # count as roots
    assert c.run(P) == -1
    c.parent[3], c.parent[5] = -1, -1
    b.rows = np.array([10, 0], np.int32)
    c.check()


def test_more_rows_than_there_are(P):
    b = Batch([8, 8], [0, 0], 16)
    c = Call(P, b, 2, 1, 128, 8)
    c.dev["row_start"].fill_(0)
    c.dev["n_rows"].fill_(16)
    assert c.run(P) == -1
    assert (f64(c.out) == 9).all()
