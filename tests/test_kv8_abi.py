"""The operators over a cache in 8 bits refuse bad arguments on the host, before
any GPU work, and so does their binding (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8

BF16, F16 = torch.bfloat16, torch.float16
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
ODD = FAKE[0] + (9 << 50) + 8


def test_append_refusals(P):
    good = P.kv8_append_config(3, 10, 8, 2, 128, 16, 40, 5, 8)
    names = ("q", "k", "v", "q_weight", "k_weight", "inv_freq", "positions", "row_start",
             "n_rows", "prefix_len", "page_table", "k_cache", "v_cache", "k_scale", "v_scale",
             "q_out", "status")

    def call(cfg, **kw):
        a = dict(zip(names, FAKE))
        a.update(kw)
        return P.LIB.pctree_kv8_append(ctypes.byref(cfg), *a.values(), None)

    for kw in (dict(batch=0), dict(total_rows=0), dict(Hq=-1), dict(Hkv=0), dict(D=0),
               dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(dtype=P.PCTREE_F32),
               dict(dtype=7), dict(rotary_dim=-16), dict(rotary_dim=144), dict(rotary_dim=24),
               dict(interleaved=2), dict(q_stride=8 * 128 - 8), dict(q_stride=8 * 128 + 4),
               dict(k_stride=2 * 128 - 8), dict(v_stride=0), dict(eps=-1.0),
               dict(eps=float("nan")), dict(rope_scale=float("inf")), dict(scale_block=0),
               dict(scale_block=3), dict(scale_block=256), dict(scale_block=-8)):
        assert call(variant(good, **kw)) == INVALID, kw
    for kw in (dict(D=96, rotary_dim=96), dict(D=256, q_stride=2048, k_stride=512, v_stride=512),
               dict(batch=1025), dict(total_rows=(1 << 30) + 1), dict(max_pages=1 << 28),
               dict(page_size=1 << 30)):
        assert call(variant(good, **kw)) == UNSUPPORTED, kw
    for name in ("q", "k", "v", "row_start", "n_rows", "prefix_len", "inv_freq", "k_cache",
                 "v_cache", "k_scale", "v_scale", "q_out"):
        assert call(good, **{name: None}) == INVALID, name
    for name in ("q", "k", "v", "q_weight", "k_weight", "k_cache", "v_cache", "q_out"):
        assert call(good, **{name: ODD}) == INVALID, name
    assert call(good, inv_freq=FAKE[5] + 4) == INVALID
    assert call(good, page_table=None) == INVALID                # no table: a page per request
    assert call(variant(good, max_pages=1, n_pages=2), page_table=None) == INVALID
    for name in ("q", "k", "v"):                                 # rows still to be read
        assert call(good, **{name: FAKE[15] + 64}) == INVALID, name
    assert P.LIB.pctree_kv8_append(None, *FAKE[:17], None) == INVALID


def test_attention_refusals(P):
    good = P.kv8_attn_config(3, 10, 8, 2, 128, 16, 40, 5, 8)
    names = ("q", "k_cache", "v_cache", "k_scale", "v_scale", "row_start", "n_rows",
             "prefix_len", "page_table", "parent", "out", "workspace")
    size = P.pctree_kv8_attention_workspace_bytes(good)
    assert size > 0 and size % 256 == 0

    def call(cfg, ws_bytes=size, **kw):
        a = dict(zip(names, FAKE))
        a.update(kw)
        return P.LIB.pctree_kv8_attention(ctypes.byref(cfg), *a.values(), ws_bytes, None, None)

    bad = [dict(batch=0), dict(total_rows=0), dict(Hq=0), dict(Hq=9), dict(Hkv=0), dict(D=0),
           dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(dtype=P.PCTREE_F32),
           dict(q_stride=8 * 128 - 8), dict(q_stride=8 * 128 + 4), dict(scale=0.0),
           dict(scale=-1.0), dict(scale=float("nan")), dict(scale_block=0), dict(scale_block=24),
           dict(scale_block=256)]
    limits = [dict(D=96), dict(D=256, q_stride=8 * 256), dict(batch=1025),
              dict(Hq=258, q_stride=258 * 128), dict(total_rows=(1 << 30) + 1),
              dict(max_pages=1 << 28)]
    for kw in bad:
        assert call(variant(good, **kw)) == INVALID, kw
    for kw in limits:
        assert call(variant(good, **kw)) == UNSUPPORTED, kw
    for kw in bad + limits:
        assert P.pctree_kv8_attention_workspace_bytes(variant(good, **kw)) == 0, kw
    for name in names[:8] + ("out",):
        assert call(good, **{name: None}) == INVALID, name
    for name in ("q", "k_cache", "v_cache", "out"):
        assert call(good, **{name: ODD}) == INVALID, name
    assert call(good, out=FAKE[0] + 256) == INVALID              # over q
    assert call(good, page_table=None) == INVALID
    assert call(good, workspace=None) == WORKSPACE
    assert call(good, workspace=FAKE[11] + 128) == WORKSPACE
    assert call(good, ws_bytes=size - 1) == WORKSPACE
    assert P.LIB.pctree_kv8_attention(None, *FAKE[:12], size, None, None) == INVALID


def test_compact_refusals(P):
    good = P.kv8_compact_config(3, 5, 16, 4, 2, 128, 16, 40, 5, 8)
    names = ("accepted_idx", "accepted_len", "prefix_len", "page_table", "k_cache", "v_cache",
             "k_scale", "v_scale", "status")

    def call(cfg, **kw):
        a = dict(zip(names, FAKE))
        a.update(kw)
        return P.LIB.pctree_kv8_compact(ctypes.byref(cfg), *a.values(), None)

    for kw in (dict(batch=0), dict(B=-1), dict(N=0), dict(layers=0), dict(Hkv=0), dict(D=0),
               dict(page_size=0), dict(n_pages=0), dict(max_pages=0), dict(scale_block=0),
               dict(scale_block=5), dict(N=81), dict(cache_layer_stride=40 * 16 * 256 - 16),
               dict(cache_layer_stride=40 * 16 * 256 + 8), dict(scale_layer_stride=40 * 2 * 2 - 1)):
        assert call(variant(good, **kw)) == INVALID, kw
    for kw in (dict(D=96), dict(D=256), dict(batch=1025), dict(max_pages=1 << 28)):
        assert call(variant(good, **kw)) == UNSUPPORTED, kw
    for name in names[:3] + names[4:8]:
        assert call(good, **{name: None}) == INVALID, name
    for name in ("k_cache", "v_cache"):
        assert call(good, **{name: ODD}) == INVALID, name
    assert call(good, page_table=None) == INVALID
    assert P.LIB.pctree_kv8_compact(None, *FAKE[:9], None) == INVALID


def test_codes_are_those_of_the_type():
    codes = np.arange(256, dtype=np.uint8)
    values = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(values, O8.VALUES, equal_nan=True)
    x = np.random.default_rng(0).standard_normal(20000) * np.exp(
        np.random.default_rng(1).uniform(-8, 4.5, 20000))
    x = np.clip(np.concatenate([x, O8.VALUES[:127], (O8.VALUES[1:127] + O8.VALUES[:126]) / 2]),
                -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(O8.encode(x), want)
    e = np.arange(112, 135, dtype=np.uint8)
    assert np.array_equal(torch.from_numpy(e).view(torch.float8_e8m0fnu).double().numpy(),
                          2.0 ** (e.astype(float) - O8.BIAS))


# ---- the binding's checks, on CPU tensors taken for those of a device -----

@pytest.fixture
def cpu(P, monkeypatch):
    """Calls whose tensors lie on the CPU reach the library's entry, which notes
    that they did."""
    monkeypatch.setattr(P, "_device_index", lambda: -1)
    monkeypatch.setattr(P, "_device_stream", lambda stream, dev: 0)
    reached = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0

    monkeypatch.setattr(P, "LIB", Lib())
    return reached


def attention_call(P):
    cfg = P.kv8_attn_config(2, 6, 4, 2, 64, 16, 5, 3, 8)
    i32 = torch.int32
    z = lambda *s, dt=BF16: torch.zeros(*s, dtype=dt)
    a = dict(q=z(6, 4, 64), k_cache=z(5, 16, 2, 64, dt=torch.uint8).view(torch.float8_e4m3fn),
             v_cache=z(5, 16, 2, 64, dt=torch.uint8),
             k_scale=z(5, 2, 2, dt=torch.uint8).view(torch.float8_e8m0fnu),
             v_scale=z(5, 2, 2, dt=torch.uint8), row_start=z(2, dt=i32), n_rows=z(2, dt=i32),
             prefix_len=z(2, dt=i32), out=z(6, 4, 64), workspace=z(1024, dt=torch.uint8),
             page_table=z(2, 3, dt=i32), parent=z(2, 3, dt=i32), status=z(1, dt=i32))
    return cfg, a


def test_binding_of_the_attention(P, cpu):
    cfg, a = attention_call(P)
    P.pctree_kv8_attention(cfg, **a)
    assert cpu == ["pctree_kv8_attention"]
    u8, i32 = torch.uint8, torch.int32
    for name, t in (("k_cache", torch.zeros(5, 16, 2, 64, dtype=BF16)),
                    ("v_cache", torch.zeros(4, 16, 2, 64, dtype=u8)),
                    ("v_cache", torch.zeros(5, 16, 64, 4, dtype=u8)[..., :2]),
                    ("k_scale", torch.zeros(5, 16, 2, dtype=u8)),        # of another block size
                    ("k_scale", torch.zeros(5, 2, 2, dtype=torch.int8)),
                    ("v_scale", torch.zeros(4, 2, 2, dtype=u8)),
                    ("v_scale", torch.zeros(5, 4, 2, dtype=u8)),
                    ("parent", torch.zeros(5, dtype=i32)),
                    ("parent", torch.zeros(2, 3, dtype=torch.int64)),
                    ("page_table", torch.zeros(2, 4, dtype=i32)),
                    ("out", torch.zeros(6, 4, 64, dtype=F16))):
        with pytest.raises(ValueError, match=name):
            P.pctree_kv8_attention(cfg, **{**a, name: t})
    P.pctree_kv8_attention(cfg, **{**a, "page_table": None, "parent": None, "status": None,
                                   "k_scale": torch.zeros(9, 2, 2, dtype=u8)})
    assert len(cpu) == 2


def test_binding_of_the_append(P, cpu):
    cfg = P.kv8_append_config(2, 6, 4, 2, 64, 16, 5, 3, 8)
    _, a = attention_call(P)
    a = {n: a[n] for n in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "row_start",
                           "n_rows", "prefix_len", "page_table")}
    a.update(k=torch.zeros(6, 2, 64, dtype=BF16), v=torch.zeros(6, 2, 64, dtype=BF16),
             q_out=torch.zeros(6, 4, 64, dtype=BF16),
             inv_freq=torch.zeros(32, dtype=torch.float64))
    P.pctree_kv8_append(cfg, **a)
    for name, t in (("k", torch.zeros(6, 3, 64, dtype=BF16)),
                    ("v_cache", torch.zeros(5, 16, 2, 64, dtype=BF16)),
                    ("k_scale", torch.zeros(5, 16, 2, dtype=torch.uint8)),
                    ("inv_freq", torch.zeros(32))):
        with pytest.raises(ValueError, match=name):
            P.pctree_kv8_append(cfg, **{**a, name: t})
    assert cpu == ["pctree_kv8_append"]


def test_binding_of_the_compaction(P, cpu):
    cfg = P.kv8_compact_config(2, 5, 16, 3, 2, 64, 16, 5, 3, 8)
    u8, i32 = torch.uint8, torch.int32
    z = lambda *s, dt=u8: torch.zeros(*s, dtype=dt)
    a = dict(accepted_idx=z(2, 6, dt=i32), accepted_len=z(2, dt=i32), prefix_len=z(2, dt=i32),
             k_cache=z(3, 5, 16, 2, 64), v_cache=z(15, 16, 2, 64), k_scale=z(3, 5, 2, 2),
             v_scale=z(3 * 5 * 4), page_table=z(2, 3, dt=i32))
    P.pctree_kv8_compact(cfg, **a)
    P.pctree_kv8_compact(cfg, **{**a, "k_cache": z(4, 5, 16, 2, 64)})
    for name, t in (("k_cache", z(3, 6, 16, 2, 64)),     # more pages than the layers' stride
                    ("k_cache", z(2, 5, 16, 2, 64)), ("k_scale", z(3, 6, 2, 2)),
                    ("v_scale", z(3, 5, 4, 2)), ("accepted_idx", z(2, 7, dt=i32))):
        with pytest.raises(ValueError, match=name):
            P.pctree_kv8_compact(cfg, **{**a, name: t})
    with pytest.raises(ValueError, match="cfg"):
        P.pctree_kv8_compact(variant(cfg, scale_layer_stride=64), **a)
    assert cpu == ["pctree_kv8_compact"] * 2
