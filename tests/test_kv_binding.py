"""What the binding of the operators around a round accepts: tensors that lie as
the call reads them, whatever their shape, and none that only have elements
enough (no GPU needed: the library's entry points are replaced)."""
import os

import pytest
import torch

BF16, I32, F32 = torch.bfloat16, torch.int32, torch.float32


@pytest.fixture()
def P(monkeypatch):
    from paper_2608_02123_gb300 import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2608_02123_gb300 import pctree
    monkeypatch.setattr(pctree, "_device_index", lambda: -1)      # of a CPU tensor
    monkeypatch.setattr(pctree, "_device_stream", lambda stream, device: 0)
    calls = []
    for name in ("pctree_kv_append", "pctree_paged_attention", "pctree_sample"):
        monkeypatch.setattr(pctree.LIB, name, lambda *a: calls.append(a) or 0)
    pctree.calls = calls
    yield pctree
    del pctree.calls


def zeros(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype)


BATCH, ROWS, HQ, HKV, D, PAGE, PAGES, MOST = 2, 6, 4, 2, 64, 16, 10, 4


def append(P, **kw):
    cfg = P.append_config(BATCH, ROWS, HQ, HKV, D, PAGE, PAGES, MOST)
    a = dict(q=zeros(ROWS, HQ, D), k=zeros(ROWS, HKV, D), v=zeros(ROWS, HKV, D),
             k_cache=zeros(PAGES, PAGE, HKV, D), v_cache=zeros(PAGES, PAGE, HKV, D),
             q_out=zeros(ROWS, HQ, D), row_start=zeros(BATCH, dtype=I32),
             n_rows=zeros(BATCH, dtype=I32), prefix_len=zeros(BATCH, dtype=I32),
             page_table=zeros(BATCH, MOST, dtype=I32), positions=zeros(ROWS, dtype=I32),
             inv_freq=zeros(D // 2, dtype=torch.float64))
    P.pctree_kv_append(cfg, **{**a, **kw})


def attention(P, **kw):
    cfg = P.paged_attn_config(BATCH, ROWS, HQ, HKV, D, PAGE, PAGES, MOST)
    a = dict(q=zeros(ROWS, HQ, D), k_cache=zeros(PAGES, PAGE, HKV, D),
             v_cache=zeros(PAGES, PAGE, HKV, D), out=zeros(ROWS, HQ, D),
             workspace=zeros(16, 8, dtype=torch.uint8), row_start=zeros(BATCH, dtype=I32),
             n_rows=zeros(BATCH, dtype=I32), prefix_len=zeros(BATCH, dtype=I32),
             page_table=zeros(BATCH, MOST, dtype=I32))
    P.pctree_paged_attention(cfg, **{**a, **kw})


TABLES = {True: [(BATCH, MOST), (BATCH + 3, MOST), (BATCH * MOST,), (1, BATCH, MOST)],
          # wider than max_pages, as allocated for the longest request; transposed
          False: [(BATCH, MOST + 1), (BATCH, 2 * MOST), (MOST, BATCH), (1, BATCH, MOST + 1),
                  (BATCH - 1, MOST)]}
CACHES = {True: [(PAGES, PAGE, HKV, D), (PAGES + 2, PAGE, HKV, D), (PAGES * PAGE, HKV, D),
                 (PAGES * PAGE + 5, HKV, D), (PAGES, PAGE, HKV * D), (PAGES * PAGE * HKV * D,),
                 (5, 2, PAGE, HKV, D), (PAGES * PAGE, HKV * D), (1, PAGES * PAGE, HKV, D)],
          # pages (or requests) further apart than page_size slots, or nearer
          False: [(PAGES, PAGE + 1, HKV, D), (PAGES, 2 * PAGE, HKV, D), (2 * PAGES, PAGE // 2, HKV, D),
                  (PAGES, PAGE, HKV + 1, D), (PAGES, PAGE, HKV, 2 * D), (PAGES - 1, PAGE, HKV, D),
                  (PAGES * PAGE, HKV + 1, D)]}
OUTS = {True: [(ROWS, HQ, D), (ROWS + 1, HQ, D), (ROWS, HQ * D), (2, 3, HQ, D),
               (ROWS * HQ * D + 3,)],
        False: [(ROWS, HQ + 1, D), (ROWS, HQ, 2 * D), (ROWS - 1, HQ, D)]}
VECTORS = {True: [(BATCH,), (BATCH + 4,), (1, BATCH + 1), (BATCH, 1)],
           False: [(BATCH, 2), (BATCH - 1,)]}


def cases(table):
    return [(good, shape) for good in (True, False) for shape in table[good]]


@pytest.mark.parametrize("call,name,dtype,good,shape", [
    (call, name, dtype, good, shape)
    for call, names in ((append, {"page_table": TABLES, "k_cache": CACHES, "v_cache": CACHES,
                                  "q_out": OUTS, "n_rows": VECTORS, "row_start": VECTORS}),
                        (attention, {"page_table": TABLES, "k_cache": CACHES, "v_cache": CACHES,
                                     "out": OUTS, "prefix_len": VECTORS}))
    for name, table in names.items()
    for dtype in (I32 if table in (TABLES, VECTORS) else BF16,)
    for good, shape in cases(table)])
def test_rows_and_caches(P, call, name, dtype, good, shape):
    t = zeros(*shape, dtype=dtype)
    if good:
        call(P, **{name: t})
        assert len(P.calls) == 1
    else:
        with pytest.raises(ValueError, match=name):
            call(P, **{name: t})
        assert not P.calls


def test_one_request_in_a_longer_contiguous_cache(P):
    cfg = P.paged_attn_config(1, ROWS, HQ, HKV, D, PAGE, 1)
    one = lambda: zeros(1, dtype=I32)
    for shape in ((1, PAGE + 9, HKV, D), (3, PAGE + 9, HKV, D)):
        P.pctree_paged_attention(cfg, zeros(ROWS, HQ, D), zeros(*shape), zeros(*shape), one(), one(),
                                 one(), zeros(ROWS, HQ, D), zeros(128, dtype=torch.uint8))
    assert len(P.calls) == 2


def test_positions_of_trees(P):
    append(P, positions=zeros(2, 3, dtype=I32))
    with pytest.raises(ValueError, match="positions must be a contiguous .* of 6 elements"):
        append(P, positions=zeros(2, 4, dtype=I32))          # rows 4 apart, not 3


def sample(P, logits, rows=6, group=3, V=40, row_stride=None, **kw):
    cfg = P.sample_config(rows, V, group, F32, row_stride)
    a = dict(uniform=zeros(rows, dtype=F32), tokens=zeros(rows, dtype=I32))
    P.pctree_sample(cfg, logits, **{**a, **kw})


def test_logits(P):
    z = lambda *s: zeros(*s, dtype=F32)
    good = [(z(6, 40), {}), (z(9, 40), {}), (z(2, 3, 40), {}), (z(4, 3, 40), {}),
            (z(6, 1, 40), {}), (z(240), dict(rows=1, group=1, V=240)),
            (z(1, 1, 40), dict(rows=1, group=1)),
            # padded vocabularies, and rows of a wider tensor
            (z(6, 48)[:, :40], dict(row_stride=48)),
            (z(2, 3, 48)[..., :40], dict(row_stride=48)),
            (z(2, 3, 48)[..., 8:], dict(row_stride=48)),
            (z(2, 6, 40)[:, ::2], dict(row_stride=80)),
            (z(5, 40), dict(rows=5)),                          # the last group cut short
            (z(2, 3, 40), dict(rows=5))]
    for t, kw in good:
        sample(P, t, **kw)
    assert len(P.calls) == len(good)
    bad = [(z(2, 4, 40), {}),                                  # rows of other nodes
           (z(2, 4, 40)[:, :3], {}),                           # groups 4 rows apart
           (z(2, 3, 48)[..., :40], {}), (z(6, 48)[:, :40], {}), (z(6, 40), dict(row_stride=48)),
           (z(5, 40), {}), (z(6, 41), {}), (z(40, 6).t(), {}), (z(6, 80)[:, ::2], {}),
           (z(3, 2, 40).transpose(0, 1), {}), (z(1, 1, 40).expand(2, 3, 40), {})]
    for t, kw in bad:
        with pytest.raises(ValueError, match="logits"):
            sample(P, t, **kw)
    assert len(P.calls) == len(good)


def test_random_numbers_and_tokens(P):
    z = zeros(6, 40, dtype=F32)
    for shape in ((6,), (8,), (2, 3), (4, 3), (6, 1)):
        sample(P, z, uniform=zeros(*shape, dtype=F32))
        sample(P, z, tokens=zeros(*shape, dtype=I32))
    for shape in ((2, 4), (5,), (3, 4)):
        with pytest.raises(ValueError, match="uniform"):
            sample(P, z, uniform=zeros(*shape, dtype=F32))
        with pytest.raises(ValueError, match="tokens"):
            sample(P, z, tokens=zeros(*shape, dtype=I32))
    for shape in ((2,), (3,), (2, 1)):
        sample(P, z, top_p=zeros(*shape, dtype=F32))
    with pytest.raises(ValueError, match="top_p"):
        sample(P, z, top_p=zeros(2, 2, dtype=F32))


def test_sample_accept_takes_logits_as_they_lie(P, monkeypatch):
    """Rows further apart than V, at N = 1 and 1 request as well."""
    seen = []
    monkeypatch.setattr(P, "pctree_sample", lambda cfg, *a: seen.append(cfg.row_stride))
    for batch, N in ((2, 3), (2, 1), (1, 3), (1, 1)):
        dr = P.Drafter.__new__(P.Drafter)
        dr.cfg = P.make_config(40, 64, 3, 2, N, batch)
        dr.target, dr.tree = None, type("T", (), {"n_nodes": None, "status": None})
        dr.accept = lambda target, stream: None
        for width in (40, 48):
            dr.sample_accept(zeros(batch, N, width, dtype=F32)[..., :40], None)
            want = width if batch * N > 1 else 40
            assert seen.pop() == want
