"""pctree_kv8_append against the float64 oracle.

Queries: pctree_kv_append's tolerance (half a step of the type and 2e-6 of the
magnitudes a rotation adds up).  Codes: half a step of the code around the
scaled value, and the same 2e-6 of those magnitudes, scaled; where nothing is
computed before the rounding (values; keys without norm and rotation) codes and
scales are the oracle's.  A key's scale is the oracle's too: inputs are drawn
so that no block's maximum lies within 1e-5 of a power of two times 448.
"""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from oracle import kv_oracle as O
from tests.kv8_util import Plane
from tests.kv_util import DTYPES, Batch, f64, half_step

pytestmark = pytest.mark.gpu

ARITHMETIC = 2e-6


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


def inv_freq(rotary, base=1e6):
    return base ** (-np.arange(0, rotary, 2, dtype=np.float64) / max(rotary, 1))


class Call:
    def __init__(self, P, b, Hq, Hkv, D, block, dtype="bf16", rotary=None, interleaved=False,
                 norm=True, positions=None, fused=True, rope_scale=1.0, seed=0, size=1.0,
                 as_bytes=False):
        self.b, self.dt, self.block = b, DTYPES[dtype], block
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, dtype=self.dt, device="cuda")
        n = b.total
        stride = None
        if fused:
            qkv = rnd(n, (Hq + 2 * Hkv) * D + 8) * size
            self.q = qkv[:, :Hq * D].unflatten(1, (Hq, D)) if Hq else None
            self.k = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
            self.v = qkv[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D].unflatten(1, (Hkv, D))
            stride = qkv.stride(0)
        else:
            self.q, self.k, self.v = (rnd(n, h, D) * size for h in (Hq, Hkv, Hkv))
        self.qw, self.kw = (rnd(D), rnd(D)) if norm else (None, None)
        self.rotary = D if rotary is None else rotary
        self.freq = inv_freq(self.rotary)
        self.pos, self.interleaved, self.rope_scale = positions, interleaved, rope_scale
        self.cfg = P.kv8_append_config(
            b.batch, n, Hq, Hkv, D, b.page_size, b.n_pages, b.max_pages, block, self.dt,
            self.rotary, interleaved, q_stride=stride, k_stride=stride, v_stride=stride,
            rope_scale=rope_scale)
        self.kp = Plane(b, Hkv, D, block, seed + 1, as_bytes=as_bytes)
        self.vp = Plane(b, Hkv, D, block, seed + 2, as_bytes=as_bytes)
        self.qo = torch.full((n + 2, max(Hq, 1), D), 9.0, dtype=self.dt, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dev = b.dev()

    def args(self):
        return dict(q=self.q, k=self.k, v=self.v, k_cache=self.kp.cache, v_cache=self.vp.cache,
                    k_scale=self.kp.scale, v_scale=self.vp.scale,
                    q_out=self.qo[1:-1] if self.q is not None else None,
                    positions=None if self.pos is None else torch.from_numpy(self.pos).cuda(),
                    inv_freq=torch.from_numpy(self.freq).cuda() if len(self.freq) else None,
                    q_weight=self.qw, k_weight=self.kw, status=self.status, **self.dev)

    def positions(self):
        b = self.b
        if self.pos is not None:
            return self.pos
        p = np.zeros(b.total, np.int64)
        for a, n, T in zip(b.start, b.rows, b.prefix):
            p[a:a + n] = T + np.arange(n)
        return p

    def want(self):
        b = self.b
        how = (self.positions(), self.freq, self.interleaved, 1e-6, self.rope_scale)
        w = {}
        weight = lambda t: None if t is None else f64(t)
        if self.q is not None:
            w["q"], w["q_size"] = O8.rotated_rows(f64(self.q), weight(self.qw), *how)
        k, w["k_size"] = O8.rotated_rows(f64(self.k), weight(self.kw), *how)
        for name, plane, x in (("k", self.kp, k), ("v", self.vp, f64(self.v))):
            codes, scales = (a[0] for a in plane.bytes())
            y = O8.append_plane(codes, scales, x, b.start, b.rows, b.prefix, b.page_size,
                                self.block, b.table)
            w[name] = (codes, scales, y)
        return w

    def run(self, P, **kw):
        P.pctree_kv8_append(self.cfg, **{**self.args(), **kw})
        torch.cuda.synchronize()
        return int(self.status.item())

    def check(self, w):
        b, u = self.b, half_step(self.dt)
        used = b.used_rows()
        if self.q is not None:
            got = f64(self.qo)
            assert (got[[0, -1]] == 9).all() and (got[1:-1][~used] == 9).all()
            tol = u * np.abs(w["q"]) + ARITHMETIC * w["q_size"] + 2.0 ** -25
            assert (np.abs(got[1:-1] - w["q"])[used] <= tol[used]).all()
        for name, plane in (("k", self.kp), ("v", self.vp)):
            codes, scales, y = w[name]
            got, got_scales = (a[0] for a in plane.bytes())
            assert (got_scales == scales).all()
            exact = name == "v" or (self.kw is None and self.rotary == 0)
            if exact:
                assert (got == codes).all()
            else:
                new = np.zeros(len(got), bool)
                for r in range(b.batch):
                    T, n, a = int(b.prefix[r]), int(b.rows[r]), int(b.start[r])
                    at = b.places(r, T, T + n)
                    new[at] = True
                    for j, p in enumerate(at):
                        s = scales[O8.block_of(T + j, r, b.page_size, self.block, b.table)]
                        e = (s.astype(int) - O8.BIAS)[:, None]
                        off = ARITHMETIC * w["k_size"][a + j] * 2.0 ** -e.astype(float)
                        want = np.clip(y[a + j], -448, 448)
                        err = np.abs(O8.VALUES[got[p]] - want)
                        assert (err <= O8.half_step(np.abs(want) + off) + off).all()
                assert (got[~new] == codes[~new]).all()
            assert plane.margins_hold()


SHAPES = {
    "token": dict(rows=[1], prefix=[2047], page=16, heads=(32, 8)),
    "tokens": dict(rows=[1] * 5, prefix=[0, 127, 128, 700, 3], page=32, heads=(40, 8)),
    "contiguous": dict(rows=[5, 0, 33], prefix=[5, 300, 129], page=0, heads=(16, 16)),
    "chains": dict(rows=[8, 8, 3, 0, 8], prefix=[100, 250, 0, 9, 121], page=32, heads=(8, 2)),
    "prompts_gaps": dict(rows=[129, 1, 64, 0, 70], prefix=[0, 40, 65, 3, 128], page=64,
                         heads=(8, 2), gap=2),
    "page_1": dict(rows=[12, 3], prefix=[20, 0], page=1, heads=(4, 2)),
    "page_23": dict(rows=[40, 17], prefix=[90, 3], page=23, heads=(4, 3)),
    "page_200": dict(rows=[150, 17], prefix=[90, 403], page=200, heads=(3, 5)),
    "no_queries": dict(rows=[30, 7], prefix=[3, 50], page=16, heads=(0, 2)),
    "one_head": dict(rows=[40, 2], prefix=[7, 60], page=48, heads=(1, 1)),
    "many_heads": dict(rows=[3], prefix=[13], page=16, heads=(70, 35)),
}


@pytest.mark.parametrize("block", [1, 2, 8, 16, 32, 128])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_shapes(P, name, block):
    s = SHAPES[name]
    b = Batch(s["rows"], s["prefix"], s["page"], gap=s.get("gap", 0))
    c = Call(P, b, *s["heads"], 128, block, seed=block)
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


@pytest.mark.parametrize("block", [1, 16])
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (64, "f16"), (128, "f16")])
@pytest.mark.parametrize("rotary,interleaved,norm", [(None, False, True), (32, True, True),
                                                     (16, False, False), (0, False, True),
                                                     (0, False, False), (None, True, False)])
def test_forms(P, D, dtype, rotary, interleaved, norm, block):
    b = Batch([21, 1, 9], [11, 40, 0], 24)
    c = Call(P, b, 4, 3, D, block, dtype, rotary=rotary, interleaved=interleaved, norm=norm,
             fused=interleaved, rope_scale=1.0 if norm else 0.75, as_bytes=norm)
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


@pytest.mark.parametrize("block", [1, 8])
def test_trees_have_given_positions(P, block):
    rng = np.random.default_rng(3)
    b = Batch([20, 13, 20], [50, 7, 90], 0)
    pos = rng.integers(0, 1 << 30, b.total).astype(np.int32)
    pos[0] = 2 ** 31 - 1
    c = Call(P, b, 8, 2, 128, block, positions=pos)
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


@pytest.mark.parametrize("block", [1, 4, 64])
@pytest.mark.parametrize("size", [1e-9, 1e-4, 30.0, 3e4])
def test_magnitudes_from_below_the_smallest_scale_to_past_the_largest(P, size, block):
    b = Batch([70, 1], [3, 0], 16)
    c = Call(P, b, 2, 2, 64, block, size=size, norm=False, rotary=0)
    c.v[0] = 0.0
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


def test_scales_at_the_borders_of_a_power_of_two(P):
    # maxima of 448 * 2^e and the next bf16 above and below it
    b = Batch([60], [0], 16)
    c = Call(P, b, 0, 1, 64, 1, norm=False, rotary=0, fused=False)
    top = 448.0 * 2.0 ** np.arange(-17, 3)
    v = np.concatenate([top, top * (1 + 2.0 ** -7), top * (1 - 2.0 ** -8)])
    c.v.zero_()
    c.v[:, 0, 5] = torch.from_numpy(v).to(c.dt).cuda()
    c.v[:, 0, 9] = -c.v[:, 0, 5] / 3
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


@pytest.mark.parametrize("block", [1, 8, 128])
def test_not_finite(P, block):
    b = Batch([20, 9], [5, 30], 16)
    c = Call(P, b, 2, 2, 64, block, norm=False, rotary=0)
    c.k[3, 1, 7] = float("nan")
    c.k[25, 0, 0] = float("inf")
    c.v[4, 0, 63] = float("-inf")
    c.v[9, 1] = float("nan")
    w = c.want()
    assert c.run(P) == -5
    c.check(w)


def test_a_query_that_is_not_finite_is_no_error(P):
    b = Batch([4], [5], 16)
    c = Call(P, b, 2, 2, 64, 1, norm=False, rotary=0)
    c.q[1, 0, 3] = float("inf")
    c.q[2, 1, 3] = float("nan")
    assert c.run(P) == 0
    assert torch.equal(c.qo[1:-1].nan_to_num(7, 8, 9), c.q.nan_to_num(7, 8, 9))


@pytest.mark.parametrize("block", [1, 16])
def test_bad_requests_and_pages(P, block):
    b = Batch([8, 8, 8, 8], [20, 3, 40, 16], 16)
    c = Call(P, b, 2, 1, 128, block)
    c.dev["n_rows"][0] = -1                              # left out
    c.dev["prefix_len"][1] = b.max_pages * b.page_size   # slots past its pages
    c.dev["page_table"][2, 2] = b.n_pages                # no page: slots 32..47
    b.rows, b.prefix = b.rows.copy(), b.prefix.copy()
    b.rows[[0, 1, 2]] = 0
    w = c.want()
    assert c.run(P) == -1
    for name, plane in (("k", c.kp), ("v", c.vp)):
        got, scales = (a[0] for a in plane.bytes())
        assert (scales == w[name][1]).all()
        if name == "v":
            assert (got == w[name][0]).all()
    got = f64(c.qo)[1:-1]
    assert (got[:16] == 9).all() and (got[16:] != 9).any()


def test_more_rows_than_there_are(P):
    b = Batch([8, 8], [0, 0], 16)
    c = Call(P, b, 2, 1, 128, 8)
    c.dev["row_start"].fill_(0)
    c.dev["n_rows"].fill_(16)
    before = c.kp.bytes()[0]
    assert c.run(P) == -1
    assert (c.kp.bytes()[0] == before).all() and (f64(c.qo) == 9).all()


def test_a_second_call_changes_nothing(P):
    b = Batch([9, 30], [21, 3], 16)
    c = Call(P, b, 2, 2, 128, 16)
    assert c.run(P) == 0
    first = [t.clone() for t in (c.kp.codes, c.kp.scales, c.vp.codes, c.vp.scales, c.qo)]
    assert c.run(P) == 0
    for t, f in zip((c.kp.codes, c.kp.scales, c.vp.codes, c.vp.scales, c.qo), first):
        assert torch.equal(t, f)


def test_values_agree_with_the_append_in_16_bits(P):
    """The same rows by pctree_kv_append: codes are those values rounded."""
    b = Batch([40, 7], [0, 0], 16)
    c = Call(P, b, 4, 2, 128, 1)
    assert c.run(P) == 0
    places = b.n_pages * b.page_size
    k16, v16 = (torch.zeros(places, 2, 128, dtype=c.dt, device="cuda") for _ in range(2))
    q16 = torch.zeros(b.total, 4, 128, dtype=c.dt, device="cuda")
    st = c.q.stride(0)
    cfg = P.append_config(b.batch, b.total, 4, 2, 128, b.page_size, b.n_pages, b.max_pages, c.dt,
                          q_stride=st, k_stride=st, v_stride=st)
    a = c.args()
    for n in ("k_scale", "v_scale"):
        a.pop(n)
    P.pctree_kv_append(cfg, **{**a, "k_cache": k16, "v_cache": v16, "q_out": q16})
    torch.cuda.synchronize()
    assert torch.equal(q16, c.qo[1:-1])
    codes, scales = (x[0] for x in c.kp.bytes())
    got = O8.values(codes, scales, b.page_size, 1)
    for r in range(b.batch):
        at = b.places(r, 0, int(b.rows[r]))
        want = f64(k16)[at]
        step = O8.half_step(want / 2.0 ** (scales[at].astype(float) - O8.BIAS)[..., None])
        tol = step * 2.0 ** (scales[at].astype(float) - O8.BIAS)[..., None] + \
            2.0 ** -8 * np.abs(want) + ARITHMETIC * 8
        assert (np.abs(got[at] - want) <= tol).all()
