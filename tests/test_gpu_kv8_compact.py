"""pctree_kv8_compact against the oracle: codes and scales are equal wherever
they are defined."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from tests.kv8_util import Plane
from tests.kv_util import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


class Call:
    def __init__(self, P, N, prefix, page, Hkv, D, block, layers, B, seed=0, lens=None,
                 exps=(-15, 7)):
        rng = np.random.default_rng(seed)
        self.b = b = Batch([N] * len(prefix), prefix, page, seed)
        self.N, self.B, self.block, self.layers = N, B, block, layers
        self.len = np.array([rng.integers(0, min(B, N - 1) + 1) for _ in prefix]
                            if lens is None else lens, np.int32)
        self.idx = np.full((b.batch, B + 1), -1, np.int32)
        for r, n in enumerate(self.len):
            self.idx[r, :n + 1] = [0] + sorted(rng.choice(np.arange(1, N), n, replace=False))
        self.kp = Plane(b, Hkv, D, block, seed + 1, layers, exps)
        self.vp = Plane(b, Hkv, D, block, seed + 2, layers, exps)
        self.cfg = P.kv8_compact_config(b.batch, B, N, layers, Hkv, D, b.page_size, b.n_pages,
                                        b.max_pages, block)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def args(self):
        d = self.b.dev()
        return dict(accepted_idx=torch.from_numpy(self.idx).cuda(),
                    accepted_len=torch.from_numpy(self.len).cuda(), prefix_len=d["prefix_len"],
                    page_table=d["page_table"], k_cache=self.kp.cache, v_cache=self.vp.cache,
                    k_scale=self.kp.scale, v_scale=self.vp.scale, status=self.status)

    def want(self, skip=()):
        b, out = self.b, []
        rows = [r for r in range(b.batch) if r not in skip]
        for plane in (self.kp, self.vp):
            codes, scales = plane.bytes()
            table = b.table
            if table is None:
                table = np.arange(b.batch, dtype=np.int32)[:, None]
            defined = [O8.compact_plane(c, s, self.idx[rows], self.len[rows], b.prefix[rows],
                                        b.page_size, self.block, table[rows])
                       for c, s in zip(codes, scales)]
            out.append((codes, scales, np.array(defined)))
        return out

    def run(self, P, **kw):
        P.pctree_kv8_compact(self.cfg, **{**self.args(), **kw})
        torch.cuda.synchronize()
        return int(self.status.item())

    def check(self, want):
        for plane, (codes, scales, defined) in zip((self.kp, self.vp), want):
            got, got_scales = plane.bytes()
            assert (got_scales == scales).all()
            assert (got[defined] == codes[defined]).all()
            assert plane.margins_hold()


@pytest.mark.parametrize("block", [1, 2, 8, 16, 32, 64, 128])
@pytest.mark.parametrize("page", [0, 1, 7, 16, 48, 200])
def test_shapes(P, page, block):
    for D, Hkv, seed in ((128, 2, 0), (64, 5, 1)):
        c = Call(P, 40, [0, 3, 17, 130], page, Hkv, D, block, 3, 16, seed)
        w = c.want()
        assert c.run(P) == 0
        c.check(w)


@pytest.mark.parametrize("block", [1, 16, 128])
def test_long_paths_and_none(P, block):
    c = Call(P, 300, [5, 100, 64, 0], 32, 1, 64, block, 2, 299, 4, lens=[299, 0, 1, 150])
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


def test_subnormal_codes_are_rounded_to_even(P):
    c = Call(P, 16, [4, 9], 16, 1, 64, 16, 1, 7, 2, lens=[5, 7], exps=(-8, -2))
    c.kp.cache.view(torch.uint8).copy_(
        torch.arange(c.kp.cache.numel()).remainder(64).to(torch.uint8).view(c.kp.cache.shape))
    w = c.want()
    assert c.run(P) == 0
    c.check(w)


def test_bad_requests_are_left_untouched(P):
    c = Call(P, 20, [4, 9, 30, 2, 8, 11, 13], 16, 2, 128, 8, 2, 6, 3, lens=[3, 3, 3, 3, 3, 3, 3])
    idx, table = c.idx.copy(), c.b.table.copy()
    w = c.want(skip=(0, 1, 2, 3, 4, 6))
    c.idx[0, 0] = 1                                  # not from the root
    c.idx[1, 2] = c.idx[1, 1]                        # not ascending
    c.idx[2, 3] = 20                                 # no node
    c.len[3] = 7                                     # longer than its row
    a = c.args()
    a["prefix_len"][4] = c.b.max_pages * c.b.page_size
    a["page_table"][6, 0] = -1
    assert c.run(P, **a) == -1
    c.check(w)


def test_one_graph_of_append_after_compact_replays(P):
    c = Call(P, 12, [5, 20], 16, 2, 64, 4, 2, 5, 9)
    a = c.args()
    w = c.want()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            P.pctree_kv8_compact(c.cfg, **a, stream=s)
        g.replay()
    s.synchronize()
    c.check(w)
