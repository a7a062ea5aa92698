"""Calls of the operators over a cache in 8 bits that the documentation allows and
that are out of the ordinary: no rows, the most requests, shared pages, several
streams, captured graphs, places past 2^32, scores of any size.  Tolerances as in
test_gpu_kv8_attention.py."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from tests.kv_util import Batch, f64, half_step
from tests.test_gpu_kv8_append import Call as Append
from tests.test_gpu_kv8_attention import Call, parents

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


@pytest.mark.parametrize("block", [1, 8])
def test_no_rows_at_all(P, block):
    b = Batch([0, 0], [4, 0], 16, gap=1)
    c = Call(P, b, 4, 2, 64, block)
    assert c.run(P) == 0
    assert (c.out == 9).all()
    a = Append(P, b, 4, 2, 64, block)
    before = a.kp.codes.clone()
    assert a.run(P) == 0
    assert torch.equal(a.kp.codes, before) and (a.qo == 9).all()


@pytest.mark.parametrize("page,rows_of", [(0, [0, 1, 1, 1, 2, 5]), (16, [0, 1, 1, 1, 2, 5]),
                                          (16, [0, 1])])
def test_as_many_requests_as_there_may_be(P, page, rows_of):
    rng = np.random.default_rng(3)
    rows = rng.choice(rows_of, 1024)
    if max(rows_of) > 1:
        rows[[0, 15, 16, 511, 512, 700, 1023]] = [70, 0, 33, 129, 40, 1, 65]
    prefix = rng.integers(0, 40, 1024)
    prefix[[3, 600]] = [300, 129]
    b = Batch(rows.tolist(), prefix.tolist(), page)
    c = Call(P, b, 4, 1, 64, 4)
    assert c.run(P) == 0
    c.check()
    a = Append(P, b, 2, 1, 64, 4, norm=False, rotary=0)
    w = a.want()
    assert a.run(P) == 0
    a.check(w)


@pytest.mark.parametrize("rows", [[1, 40, 3], [1, 1, 1]])
def test_requests_that_share_the_pages_of_a_prefix(P, rows):
    b = Batch(rows, [100, 130, 96], 16)
    b.table[1, :6] = b.table[0, :6]
    b.table[2, :6] = b.table[0, :6]
    c = Call(P, b, 8, 2, 128, 16)
    assert c.run(P) == 0
    c.check()


def test_one_long_request_among_tokens(P):
    """Units of one row, of a request that has many."""
    b = Batch([1, 1, 30, 0, 0, 0] + [0] * 40, [10, 200, 300, 0, 5, 1] + [0] * 40, 16)
    c = Call(P, b, 8, 2, 128, 2)
    assert c.run(P) == 0
    c.check()


def test_two_calls_at_once(P):
    calls = [Call(P, Batch([1] * 20, [int(x) for x in range(5, 1005, 50)], 64), 16, 4, 128),
             Call(P, Batch([205, 300], [40, 7], 16, seed=1), 16, 2, 128, 4, seed=1),
             Call(P, Batch([30, 90], [0, 333], 48, seed=2), 16, 2, 64, 16, "f16", seed=2)]
    calls[2].parent = parents(calls[2].b)
    want = [c.want() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(calls, streams):
            P.pctree_kv8_attention(c.cfg, **c.args(), stream=s)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert int(c.status.item()) == 0
        c.check(w)


@pytest.mark.parametrize("rows", [[70, 1, 9], [1, 1, 1]])
def test_streams_and_graphs(P, rows):
    """On another stream, and replayed from two graphs that share a workspace
    one after the other."""
    b = Batch(rows, [5, 900, 20], 16)
    c = Call(P, b, 8, 2, 128)
    want = c.want()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.pctree_kv8_attention(c.cfg, **c.args(), stream=s)
    torch.cuda.synchronize()
    c.check(want)
    d = Call(P, b, 8, 2, 128, seed=5)
    d.ws = c.ws
    graphs, held = [], []
    for x in (c, d):
        g = torch.cuda.CUDAGraph()
        args = x.args()
        held.append(args)
        with torch.cuda.graph(g, stream=s):
            P.pctree_kv8_attention(x.cfg, **args)
        graphs.append(g)
    for _ in range(3):
        c.out.fill_(9)
        d.out.fill_(9)
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    c.check(want)
    d.check()


@pytest.mark.parametrize("rows", [[20, 1], [1, 1]])
def test_peaked_and_growing_scores(P, rows):
    """Maxima that grow along the keys move every row's reference, and scores far
    apart leave one key.  Scores of up to 119, after the float32 sum of 128 equal
    terms: 128 * 2^-24 of them absolute, 9.1e-4; of a probability twice."""
    b = Batch(rows, [400, 300], 16)
    for factor in (0.02, 12.0):
        c = Call(P, b, 4, 2, 128, garbage=False)
        places = b.n_pages * b.page_size
        c.q.zero_().add_(factor)
        order = np.zeros(places, np.int64)
        for r in range(2):
            at = b.places(r, 0, int(b.prefix[r] + b.rows[r]))
            order[at] = np.arange(len(at)) * 126 // len(at)
        codes = torch.from_numpy(order.astype(np.uint8)).cuda()
        c.kp.cache.view(torch.uint8).view(places, 2, 128).copy_(codes[:, None, None])
        c.kp.scale.view(torch.uint8).fill_(127 - 9)
        assert c.run(P) == 0
        out, size = c.want()
        got, u = f64(c.out[1:-1]), half_step(c.dt)
        tol = (2.0 ** -11 + 2 * 9.2e-4 + 5e-4) * size + u * np.abs(out)
        assert (np.abs(got - out) <= tol).all()


@pytest.mark.parametrize("rows", [[40, 1], [1, 1]])
@pytest.mark.parametrize("size", [3e6, 1e8, -1e8])
def test_scores_whose_floats_are_far_apart(P, rows, size):
    """Equal scores past 2^22 (in log2 units) are equal probabilities, and one
    score a step above them is the only one left."""
    b = Batch(rows, [300, 70], 16)
    for one in (False, True):
        c = Call(P, b, 4, 2, 128, garbage=False)
        places = b.n_pages * b.page_size
        c.cfg.scale = 1.0
        c.q.zero_()
        c.q[:, :, 3] = size
        k = c.kp.cache.view(torch.uint8).view(places, 2, 128)
        k.zero_()
        k[:, :, 3] = int(O8.encode(1.0))
        c.kp.scale.view(torch.uint8).fill_(127)
        if one:
            k[int(b.places(0, 17, 18)[0]), :, 3] = int(O8.encode(1.125 if size > 0 else 0.875))
        assert c.run(P) == 0
        c.check()


def test_a_row_whose_query_is_not_finite_is_nan_alone(P):
    for rows in ([20, 3], [1, 1]):
        b = Batch(rows, [50, 200], 16)
        for value in (float("nan"), float("inf")):
            c = Call(P, b, 4, 2, 128)
            c.q[0, 1, 5] = value
            assert c.run(P) == 0
            got = f64(c.out)[1:-1]
            assert np.isnan(got[0, 1]).all()
            got[0, 1] = 0.0
            assert np.isfinite(got).all()


def test_places_past_32_bits(P):
    """Append, attention and compaction in the last pages of a cache whose planes
    have more than 2^32 bytes."""
    Hkv, D, page, block, N = 64, 128, 64, 8, 8
    pages = (1 << 32) // (Hkv * D * page) + 4
    u8 = dict(dtype=torch.uint8, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros(pages, page, Hkv, D, **u8) for _ in range(2))
    ks, vs = (torch.full((pages, page // block, Hkv), 127, **u8) for _ in range(2))
    table = torch.tensor([[pages - 1, 3, pages - 2]], **i32)
    n = 3 * page - 17
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.bfloat16, device="cuda")
    k, v = rnd(n, Hkv, D), rnd(n, Hkv, D)
    zero = torch.zeros(1, **i32)
    cfg = P.kv8_append_config(1, n, 0, Hkv, D, page, pages, 3, block, rotary_dim=0)
    P.pctree_kv8_append(cfg, None, k, v, kc, vc, ks, vs, None, zero, torch.full((1,), n, **i32),
                        zero, page_table=table)
    order = [pages - 1, 3, pages - 2]
    seen = lambda c, s: (c[order].view(torch.float8_e4m3fn).double().view(-1, Hkv, D)
                         * s[order].view(torch.float8_e8m0fnu).double()
                         .repeat_interleave(block, 1).view(-1, Hkv)[..., None])
    K, V = seen(kc, ks), seen(vc, vs)
    top = k.double().abs().view(-1, Hkv, D)[:n - n % block].unflatten(0, (-1, block)).amax((1, 3))
    step = top.repeat_interleave(block, 0)[..., None] * 2.0 ** -4
    assert bool(((K[:n - n % block] - k[:n - n % block].double()).abs() <= step).all())
    for rows in (1, 40):
        q = rnd(rows, Hkv, D)
        cfg = P.kv8_attn_config(1, rows, Hkv, Hkv, D, page, pages, 3, block)
        ws = torch.empty(P.pctree_kv8_attention_workspace_bytes(cfg), **u8)
        out = torch.empty_like(q)
        P.pctree_kv8_attention(cfg, q, kc, vc, ks, vs, zero, torch.full((1,), rows, **i32),
                               torch.full((1,), n - rows, **i32), out, ws, page_table=table)
        s = torch.einsum("hd,shd->hs", q[-1].double(), K[:n]) * D ** -0.5
        p = s.softmax(-1)
        want = torch.einsum("hs,shd->hd", p, V[:n])
        size = torch.einsum("hs,shd->hd", p, V[:n].abs())
        u = half_step(torch.bfloat16)
        tol = (2.0 ** -11 + 5e-4) * size + u * want.abs() + n * 2.0 ** -32 * 8
        assert bool(((out[-1].double() - want).abs() <= tol).all())
    T = n - N
    before_k, before_s = kc[order].clone(), ks[order].clone()
    cc = P.kv8_compact_config(1, 3, N, 1, Hkv, D, page, pages, 3, block)
    P.pctree_kv8_compact(cc, torch.tensor([[0, 2, 5, -1]], **i32), torch.tensor([2], **i32),
                         torch.tensor([T], **i32), kc, vc, ks, vs, page_table=table)
    got = seen(kc, ks)
    was = (before_k.view(torch.float8_e4m3fn).double().view(-1, Hkv, D)
           * before_s.view(torch.float8_e8m0fnu).double().repeat_interleave(block, 1)
           .view(-1, Hkv)[..., None])
    # (a code may lose its lowest bit where it becomes subnormal: 2^-10 of the scale)
    room = 2.0 ** -10 * ks[order].view(torch.float8_e8m0fnu).double().repeat_interleave(
        block, 1).view(-1, Hkv)[..., None]
    for j, a in enumerate([0, 2, 5]):
        assert bool(((got[T + j] - was[T + a]).abs() <= room[T + j]).all())
    assert torch.equal(kc[order].view(-1, Hkv, D)[:T - T % block],
                       before_k.view(-1, Hkv, D)[:T - T % block])
