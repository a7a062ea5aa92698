"""The operators around a round refuse bad arguments on the host, before any
GPU work (no GPU needed)."""
import ctypes
import os

import pytest
import torch

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INVALID, WORKSPACE, UNSUPPORTED = -1, -2, -6


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import build
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2608_02123_gb300 import pctree
    return pctree


def variant(cfg, **kw):
    f = {n: getattr(cfg, n) for n, _ in cfg._fields_}
    f.update(kw)
    return type(cfg)(**f)


# one 16-byte aligned fake address per argument, far apart
FAKE = [(i + 1) << 40 for i in range(20)]


def test_append_refusals(P):
    good = P.append_config(3, 10, 8, 2, 128, 16, 40, 5)
    names = ("q", "k", "v", "q_weight", "k_weight", "inv_freq", "positions", "row_start",
             "n_rows", "prefix_len", "page_table", "k_cache", "v_cache", "q_out", "status")

    def call(cfg, **kw):
        a = dict(zip(names, FAKE))
        a.update(kw)
        return P.LIB.pctree_kv_append(ctypes.byref(cfg), *a.values(), None)

    for kw in (dict(batch=0), dict(total_rows=0), dict(Hq=-1), dict(Hkv=0), dict(D=0),
               dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(dtype=P.PCTREE_F32),
               dict(dtype=7), dict(rotary_dim=-16), dict(rotary_dim=144), dict(rotary_dim=24),
               dict(interleaved=2), dict(q_stride=8 * 128 - 8), dict(q_stride=8 * 128 + 4),
               dict(k_stride=2 * 128 - 8), dict(v_stride=0), dict(eps=-1.0),
               dict(eps=float("nan")), dict(rope_scale=float("inf"))):
        assert call(variant(good, **kw)) == INVALID, kw
    for kw in (dict(D=96, rotary_dim=96), dict(batch=1025), dict(total_rows=(1 << 30) + 1),
               dict(max_pages=1 << 28), dict(page_size=1 << 30)):
        assert call(variant(good, **kw)) == UNSUPPORTED, kw
    for name in ("q", "k", "v", "row_start", "n_rows", "prefix_len", "inv_freq", "k_cache",
                 "v_cache", "q_out"):
        assert call(good, **{name: None}) == INVALID, name
    for name in ("q", "k", "v", "q_weight", "k_weight", "k_cache", "v_cache", "q_out"):
        assert call(good, **{name: FAKE[0] + (9 << 50) + 8}) == INVALID, name
    assert call(good, inv_freq=FAKE[5] + 4) == INVALID
    # no table: a page per request
    assert call(good, page_table=None) == INVALID
    assert call(variant(good, max_pages=1, n_pages=2), page_table=None) == INVALID
    # q_out over rows that are still to be read
    for name in ("q", "k", "v"):
        assert call(good, **{name: FAKE[13] + 64}) == INVALID, name
    assert P.LIB.pctree_kv_append(None, *FAKE[:15], None) == INVALID


def test_paged_attention_refusals(P):
    good = P.paged_attn_config(3, 10, 8, 2, 128, 16, 40, 5)
    names = ("q", "k_cache", "v_cache", "row_start", "n_rows", "prefix_len", "page_table", "out",
             "workspace")
    size = P.pctree_paged_attention_workspace_bytes(good)
    assert size > 0 and size % 256 == 0

    def call(cfg, ws_bytes=size, **kw):
        a = dict(zip(names, FAKE))
        a.update(kw)
        return P.LIB.pctree_paged_attention(ctypes.byref(cfg), *a.values(), ws_bytes, None, None)

    bad = [dict(batch=0), dict(total_rows=0), dict(Hq=0), dict(Hq=9), dict(Hkv=0), dict(D=0),
           dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(dtype=P.PCTREE_F32),
           dict(q_stride=8 * 128 - 8), dict(q_stride=8 * 128 + 4), dict(scale=0.0),
           dict(scale=-1.0), dict(scale=float("nan"))]
    limits = [dict(D=96), dict(D=256, q_stride=8 * 256), dict(batch=1025),
              dict(Hq=258, q_stride=258 * 128), dict(total_rows=(1 << 30) + 1),
              dict(max_pages=1 << 28)]
    for kw in bad:
        assert call(variant(good, **kw)) == INVALID, kw
    for kw in limits:
        assert call(variant(good, **kw)) == UNSUPPORTED, kw
    for kw in bad + limits:
        assert P.pctree_paged_attention_workspace_bytes(variant(good, **kw)) == 0, kw
    for name in names[:6] + ("out",):
        assert call(good, **{name: None}) == INVALID, name
    for name in ("q", "k_cache", "v_cache", "out"):
        assert call(good, **{name: FAKE[0] + (9 << 50) + 8}) == INVALID, name
    assert call(good, out=FAKE[0] + 256) == INVALID            # over q
    assert call(good, page_table=None) == INVALID
    assert call(good, workspace=None) == WORKSPACE
    assert call(good, workspace=FAKE[8] + 128) == WORKSPACE
    assert call(good, ws_bytes=size - 1) == WORKSPACE
    assert P.LIB.pctree_paged_attention(None, *FAKE[:9], size, None, None) == INVALID


def test_sample_refusals(P):
    good = P.sample_config(4, 1000, 2, BF16)

    def call(cfg, logits=FAKE[0], uniform=FAKE[1], tokens=FAKE[2]):
        return P.LIB.pctree_sample(ctypes.byref(cfg), logits, uniform, None, None, None, None,
                                   None, tokens, None, None)

    for kw in (dict(rows=0), dict(V=0), dict(group=0), dict(dtype=3), dict(dtype=-1),
               dict(row_stride=999)):
        assert call(variant(good, **kw)) == INVALID, kw
    for kw in (dict(V=(1 << 18) + 1, row_stride=1 << 19), dict(rows=(1 << 27) + 1),
               dict(row_stride=(1 << 40) + 1)):
        assert call(variant(good, **kw)) == UNSUPPORTED, kw
    assert call(good, logits=None) == INVALID
    assert call(good, uniform=None) == INVALID
    assert call(good, tokens=None) == INVALID
    assert call(good, logits=FAKE[0] + 1) == INVALID
    assert P.LIB.pctree_sample(None, *FAKE[:10]) == INVALID


def test_oracle_sample_row():
    """The sampling oracle on rows worked out by hand."""
    import numpy as np
    from oracle.kv_oracle import sample_row
    z = np.log(np.array([1.0, 4.0, 2.0, 1.0]) / 8)
    assert [sample_row(z, u) for u in (0.0, 0.124, 0.126, 0.624, 0.626, 0.874, 0.876)] == \
        [0, 0, 1, 1, 2, 2, 3]
    assert sample_row(z, 0.99, temperature=0.0) == 1
    assert [sample_row(z, u, top_k=2) for u in (0.0, 0.66, 0.67)] == [1, 1, 2]
    # ties: the lowest index of the two ones is kept
    assert [sample_row(z, u, top_k=3) for u in (0.14, 0.15)] == [0, 1]
    assert [sample_row(z, u, top_p=0.49) for u in (0.0, 0.99)] == [1, 1]
    assert [sample_row(z, u, top_p=0.51) for u in (0.66, 0.67)] == [1, 2]
    assert [sample_row(z, u, min_p=0.4) for u in (0.66, 0.67)] == [1, 2]
    # temperature 1/2 squares the weights: 1, 16, 4, 1
    assert [sample_row(z, u, temperature=0.5) for u in (0.045, 0.046, 0.772, 0.773)] == [0, 1, 1, 2]
    # top-p counts what top-k left: 4 of 6 reaches 0.6
    assert sample_row(z, 0.99, top_k=2, top_p=0.6) == 1


def test_oracle_norm_rotate():
    """The append oracle against complex multiplication."""
    import numpy as np
    from oracle.kv_oracle import norm_rotate
    rng = np.random.default_rng(0)
    x, w, f = rng.normal(size=8), rng.normal(size=8), np.array([1.0, 0.25])
    for interleaved in (False, True):
        y, _ = norm_rotate(x, w, 3, f, interleaved, 0.0)
        n = x * w / np.sqrt(np.mean(x * x))
        a, b = ([0, 2], [1, 3]) if interleaved else ([0, 1], [2, 3])
        z = (n[a] + 1j * n[b]) * np.exp(3j * f)
        assert np.allclose(y[a], z.real) and np.allclose(y[b], z.imag)
        assert np.allclose(y[4:], n[4:])


def test_oracle_paged_attention_follows_the_table():
    """Paged and contiguous storage of the same slots give the same rows, and
    a later key changes no earlier row."""
    import numpy as np
    from oracle.kv_oracle import paged_attention
    rng = np.random.default_rng(1)
    q, K, V = rng.normal(size=(3, 4, 8)), rng.normal(size=(12, 2, 8)), rng.normal(size=(12, 2, 8))
    a, _ = paged_attention(q, K, V, [0], [3], [5], 12, None, 0.3)
    order = np.array([3, 1, 0, 2])
    Kp, Vp = np.zeros((20, 2, 8)), np.zeros((20, 2, 8))
    for i, p in enumerate(order[:3]):
        Kp[p * 4:p * 4 + 4], Vp[p * 4:p * 4 + 4] = K[i * 4:i * 4 + 4], V[i * 4:i * 4 + 4]
    b, _ = paged_attention(q, Kp, Vp, [0], [3], [5], 4, order[None], 0.3)
    assert np.allclose(a, b)
    K[7] = 50.0
    c, _ = paged_attention(q, K, V, [0], [3], [5], 12, None, 0.3)
    assert np.allclose(a[:2], c[:2]) and not np.allclose(a[2], c[2])
