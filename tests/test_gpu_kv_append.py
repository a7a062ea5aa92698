"""pctree_kv_append against the float64 oracle.

Tolerance per element y = a cos t - b sin t (size = |a| + |b|): one rounding to
the type, half a step of |y|; before it float32 arithmetic: the norm's sum of
at most 256 squares (16 in a lane, then a tree: at most 20 additions, 2^-24
each, halved by the root), rsqrt (2 ulp), three products, the sine and cosine
(2 ulp and an angle rounded to 2^-25 of a half turn: below 4e-7 absolute) and
the final difference: below 2e-6 * size together.  Values and heads without
norm or rotation are copies.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
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
    """One call's tensors, with margins of a fixed pattern."""

    def __init__(self, P, b, Hq, Hkv, D, dtype="bf16", rotary=None, interleaved=False, norm=True,
                 positions=None, fused=True, eps=1e-6, rope_scale=1.0, seed=0):
        self.b, self.dt = b, DTYPES[dtype]
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, dtype=self.dt, device="cuda")
        n = b.total
        if fused:
            qkv = rnd(n, (Hq + 2 * Hkv) * D + 8)
            self.q = qkv[:, :Hq * D].unflatten(1, (Hq, D)) if Hq else None
            self.k = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
            self.v = qkv[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D].unflatten(1, (Hkv, D))
            stride = qkv.stride(0)
        else:
            self.q, self.k, self.v = (rnd(n, h, D) for h in (Hq, Hkv, Hkv))
            stride = None
        self.qw, self.kw = (rnd(D), rnd(D)) if norm else (None, None)
        rotary = D if rotary is None else rotary
        self.freq = inv_freq(rotary)
        self.pos = positions
        self.cfg = P.append_config(b.batch, n, Hq, Hkv, D, b.page_size, b.n_pages, b.max_pages,
                                   self.dt, rotary, interleaved, q_stride=stride,
                                   k_stride=stride, v_stride=stride, eps=eps,
                                   rope_scale=rope_scale)
        places = b.n_pages * b.page_size
        self.kc = torch.full((places + 2, Hkv, D), 7.0, dtype=self.dt, device="cuda")
        self.vc = torch.full((places + 2, Hkv, D), -7.0, dtype=self.dt, device="cuda")
        self.qo = torch.full((n + 2, max(Hq, 1), D), 9.0, dtype=self.dt, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.dev = b.dev()

    def args(self):
        b = self.b
        return dict(q=self.q, k=self.k, v=self.v, k_cache=self.kc[1:-1], v_cache=self.vc[1:-1],
                    q_out=self.qo[1:-1] if self.q is not None else None,
                    positions=None if self.pos is None else
                    torch.from_numpy(self.pos).cuda(),
                    inv_freq=torch.from_numpy(self.freq).cuda() if len(self.freq) else None,
                    q_weight=self.qw, k_weight=self.kw, status=self.status, **self.dev)

    def run(self, P, **kw):
        P.pctree_kv_append(self.cfg, **{**self.args(), **kw})
        torch.cuda.synchronize()
        return int(self.status.item())

    def check(self, skip=()):
        b, cfg = self.b, self.cfg
        u = half_step(self.dt)
        tiny = 2.0 ** -25 if self.dt is torch.float16 else 0.0     # half a subnormal step
        kc, vc, qo = f64(self.kc), f64(self.vc), f64(self.qo)
        k, v = f64(self.k), f64(self.v)
        q = None if self.q is None else f64(self.q)
        qw, kw = (None if w is None else f64(w) for w in (self.qw, self.kw))
        seen_k = np.zeros(len(kc), bool)
        seen_q = np.zeros(len(qo), bool)

        def close(got, x, w, pos):
            want, size = O.norm_rotate(x, w, pos, self.freq, cfg.interleaved, cfg.eps,
                                       cfg.rope_scale)
            err = ARITHMETIC * size if (w is not None or len(self.freq)) else 0.0 * size
            assert (np.abs(got - want) <= u * (np.abs(want) + err) + err + tiny).all()

        for r in range(b.batch):
            for j in range(int(b.rows[r])):
                i, slot = int(b.start[r]) + j, int(b.prefix[r]) + j
                pos = slot if self.pos is None else int(self.pos[i])
                if q is not None:
                    seen_q[1 + i] = True
                    for h in range(cfg.Hq):
                        close(qo[1 + i, h], q[i, h], qw, pos)
                if (r, j) in skip:
                    continue
                at = 1 + O.place_of(slot, r, b.page_size, b.table)
                assert not seen_k[at]
                seen_k[at] = True
                np.testing.assert_array_equal(vc[at], v[i])
                for h in range(cfg.Hkv):
                    close(kc[at, h], k[i, h], kw, pos)
        # every other place and row is as it was
        assert (kc[~seen_k] == 7).all() and (vc[~seen_k] == -7).all()
        assert (qo[~seen_q] == 9).all()


SHAPES = {
    "one_token": dict(rows=[1], prefix=[0], page=16, heads=(32, 8), D=128),
    "one_token_far": dict(rows=[1], prefix=[2047], page=16, heads=(32, 8), D=128),
    "ragged": dict(rows=[5, 0, 33, 1], prefix=[0, 4, 17, 64], page=8, heads=(10, 2), D=64, gap=3),
    "contiguous": dict(rows=[7, 12], prefix=[3, 0], page=0, heads=(5, 5), D=128, gap=1),
    "odd_pages": dict(rows=[70, 3], prefix=[1, 46], page=23, heads=(4, 1), D=256),
    "one_row_pages": dict(rows=[9, 2], prefix=[1, 6], page=1, heads=(3, 3), D=64),
    "many_rows": dict(rows=[611, 300], prefix=[9, 2], page=64, heads=(2, 1), D=64),
    "many_requests": dict(rows=[1] * 70, prefix=list(range(70)), page=16, heads=(2, 2), D=64),
    "no_queries": dict(rows=[6, 4], prefix=[0, 9], page=32, heads=(0, 3), D=128),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", sorted(SHAPES))
def test_shapes(P, name, dtype):
    s = SHAPES[name]
    b = Batch(s["rows"], s["prefix"], s["page"], gap=s.get("gap", 0))
    c = Call(P, b, *s["heads"], s["D"], dtype)
    assert c.run(P) == 0
    c.check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rotary", [0, 16, 32, "half", "all"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotation_forms(P, D, rotary, interleaved, norm):
    rotary = {"half": D // 2, "all": D}.get(rotary, rotary)
    b = Batch([4, 3], [11, 30], 16)
    c = Call(P, b, 6, 2, D, "bf16" if norm else "f16", rotary, interleaved, norm,
             fused=interleaved, rope_scale=1.0 if norm else 0.75)
    assert c.run(P) == 0
    c.check()


def test_given_positions_far_and_negative(P):
    b = Batch([6, 3], [2, 5], 16, gap=2)
    pos = np.full(b.total, -1, np.int32)
    pos[:6] = [0, 1, 1, 1_000_003, 2**31 - 1, -12345]
    pos[8:11] = [131071, 131072, 16777217]
    c = Call(P, b, 4, 2, 128, positions=pos)
    assert c.run(P) == 0
    c.check()


def test_zero_rows_and_zero_heads(P):
    """A row of zeros stays zero under a norm with eps, and is NaN without
    (0 * rsqrt(0))."""
    b = Batch([3], [4], 16)
    c = Call(P, b, 2, 1, 64, fused=False)
    c.q.zero_()
    c.k.zero_()
    assert c.run(P) == 0
    assert not c.qo[1:-1].any()
    c.check()


def test_bad_requests_and_pages(P):
    b = Batch([3, 4, 2, 5], [4, 0, 30, 7], 8)
    good = b.table.copy()
    # request 1's page 0 is no page; request 3's rows end past the row tensors
    b.table[1, 0] = b.n_pages
    c = Call(P, b, 4, 2, 64)
    assert c.run(P) == -1
    b.table[1, 0] = good[1, 0]
    c.check(skip={(1, j) for j in range(4)})
    for name, value in (("prefix_len", -1), ("prefix_len", b.max_pages * 8 - 4),
                        ("n_rows", -1), ("n_rows", 6), ("row_start", -1),
                        ("row_start", b.total - 4)):
        c = Call(P, b, 4, 2, 64)
        c.dev[name][3] = value
        assert c.run(P) == -1, name
        keep = b.rows.copy()
        b.rows[3] = 0                              # as if the request had no rows
        c.check()
        b.rows[:] = keep


def test_other_stream_and_graph_replay(P):
    b = Batch([40, 3], [5, 20], 16)
    c = Call(P, b, 8, 2, 128)
    args = c.args()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.pctree_kv_append(c.cfg, **args, stream=s)
    torch.cuda.synchronize()
    c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        P.pctree_kv_append(c.cfg, **args)
    for t, x in ((c.kc, 7.0), (c.vc, -7.0), (c.qo, 9.0)):
        t.fill_(x)
    g.replay()
    torch.cuda.synchronize()
    c.check()


def test_places_past_32_bits(P):
    """A cache of more than 2^32 elements: rows in its last pages."""
    Hkv, D, page = 64, 256, 64
    pages = (1 << 32) // (Hkv * D * page) + 2
    kc = torch.zeros(pages, page, Hkv, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    k = torch.randn(2, Hkv, D, dtype=torch.bfloat16, device="cuda")
    v = torch.randn_like(k)
    i32 = dict(dtype=torch.int32, device="cuda")
    cfg = P.append_config(1, 2, 0, Hkv, D, page, pages, 2, rotary_dim=0)
    P.pctree_kv_append(cfg, None, k, v, kc, vc, None, torch.zeros(1, **i32),
                       torch.full((1,), 2, **i32), torch.full((1,), page - 1, **i32),
                       page_table=torch.tensor([[pages - 1, pages - 2]], **i32))
    assert torch.equal(kc[pages - 1, page - 1], k[0]) and torch.equal(kc[pages - 2, 0], k[1])
    assert torch.equal(vc[pages - 1, page - 1], v[0]) and torch.equal(vc[pages - 2, 0], v[1])
    assert int(kc.count_nonzero()) == int(k.count_nonzero())
