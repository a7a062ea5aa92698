"""Oracles of the operators over a cache in 8 bits.  TEST INFRASTRUCTURE ONLY.

Plain float64 restatements, request by request, of what ``include/pctree.h`` says
of ``pctree_kv8_append``, ``pctree_kv8_attention`` and ``pctree_kv8_compact``.
They share no code with the CUDA library.
"""
from __future__ import annotations

import numpy as np

from .kv_oracle import norm_rotate, place_of

MIN_EXP, MAX_EXP, BIAS = -15, 7, 127


def _table():
    t = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if (c & 127) == 127:
            v = np.nan
        t[c] = -v if c & 128 else v
    return t


VALUES = _table()                    # of the codes
_LADDER = VALUES[:127]               # ascending, 0 .. 448


def half_step(y):
    """Half the distance of the codes around |y| (of the largest past 448)."""
    y = np.minimum(np.abs(y), 448.0)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.where(y > 0, y, 1e-300)))
    return 2.0 ** (np.maximum(e, -6.0) - 4.0)


def encode(y):
    """Codes of float64 values: to nearest, ties to the even code; past 448 the
    largest; 0x7f (NaN) for what is not finite."""
    y = np.asarray(y, np.float64)
    a = np.minimum(np.where(np.isfinite(y), np.abs(y), 0.0), 448.0)
    hi = np.clip(np.searchsorted(_LADDER, a), 1, 126)
    lo = hi - 1
    d = (a - _LADDER[lo]) - (_LADDER[hi] - a)
    c = np.where(d < 0, lo, np.where(d > 0, hi, np.where(lo % 2 == 0, lo, hi)))
    c = c | np.where(np.signbit(y), 128, 0)
    return np.where(np.isfinite(y), c, 127).astype(np.uint8)


def least_exp(top):
    """The smallest exponent of the range with 448 * 2^e >= top."""
    e = np.full(np.shape(top), MAX_EXP)
    for x in range(MAX_EXP, MIN_EXP - 1, -1):
        e = np.where(448.0 * 2.0 ** x >= top, x, e)
    return e


def block_of(slot, r, page_size, block, table):
    """Place of a slot's scale in [n_pages * ceil(page_size / block)]."""
    page = r if table is None else int(table[r][slot // page_size])
    return page * -(-page_size // block) + slot % page_size // block


def append_plane(codes, scales, x, start, rows, prefix, page_size, block, table):
    """Appends x [total][Hkv][D] (float64, after norm and rotation) to codes
    [places][Hkv][D] uint8 and scales [blocks][Hkv] uint8, in place.  Returns the
    scaled values [total][Hkv][D] that were rounded (NaN in rows of no request)."""
    scaled = np.full(x.shape, np.nan)
    for r in range(len(rows)):
        T, n, a = int(prefix[r]), int(rows[r]), int(start[r])
        by_block = {}
        for j in range(n):
            by_block.setdefault(block_of(T + j, r, page_size, block, table), []).append(j)
        for at, js in by_block.items():
            new = x[a + np.array(js)]
            size = np.where(np.isfinite(new), np.abs(new), 0.0)
            e = least_exp(size.max(axis=(0, 2)))
            before = [s for s in range(max(0, T - block), T)
                      if block_of(s, r, page_size, block, table) == at]
            if before:
                old = scales[at].astype(int) - BIAS
                e = np.maximum(e, old)
                for s in before:
                    p = place_of(s, r, page_size, table)
                    codes[p] = encode(VALUES[codes[p]] * 2.0 ** (old - e)[:, None])
            scales[at] = e + BIAS
            for j in js:
                y = x[a + j] * 2.0 ** -e[:, None].astype(np.float64)
                scaled[a + j] = y
                codes[place_of(T + j, r, page_size, table)] = encode(y)
    return scaled


def rotated_rows(x, weight, positions, inv_freq, interleaved, eps, rope_scale=1.0):
    """x [rows][heads][D] normed and rotated, and each element's magnitudes."""
    out, size = np.zeros(x.shape), np.zeros(x.shape)
    for i in range(x.shape[0]):
        for h in range(x.shape[1]):
            out[i, h], size[i, h] = norm_rotate(x[i, h], weight, positions[i], inv_freq,
                                                interleaved, eps, rope_scale)
    return out, size


def values(codes, scales, page_size, block):
    """The cache's values [places][Hkv][D]."""
    places = np.arange(codes.shape[0])
    at = places // page_size * -(-page_size // block) + places % page_size // block
    return VALUES[codes] * 2.0 ** (scales[at].astype(np.float64) - BIAS)[..., None]


def sees(j, T, parent):
    """Slots that row j of a request sees: causal, or its path in the tree."""
    if parent is None:
        return np.arange(T + j + 1)
    path = []
    while j >= 0:
        path.append(T + j)
        j = int(parent[j])
    return np.concatenate([np.arange(T), path[::-1]]).astype(np.int64)


def attention(q, K, V, row_start, n_rows, prefix_len, page_size, table, scale, parent=None):
    """q [rows][Hq][D], K / V [places][Hkv][D] float64, parent [rows] or None.
    Returns out (NaN in rows of no request) and sum_s p_s |v_s| beside it."""
    rows, Hq, D = q.shape
    G = Hq // K.shape[1]
    out, size = np.full((rows, Hq, D), np.nan), np.zeros((rows, Hq, D))
    for r in range(len(n_rows)):
        T, n, a = int(prefix_len[r]), int(n_rows[r]), int(row_start[r])
        at = np.array([place_of(s, r, page_size, table) for s in range(T + n)], np.int64)
        for j in range(n):
            see = at[sees(j, T, None if parent is None else parent[a:a + n])]
            for h in range(Hq):
                k, v = K[see, h // G], V[see, h // G]
                with np.errstate(invalid="ignore"):
                    s = scale * (k @ q[a + j, h])
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[a + j, h], size[a + j, h] = p @ v, p @ np.abs(v)
    return out, size


def compact_plane(codes, scales, idx, length, prefix, page_size, block, table):
    """Moves the accepted rows in codes [places][Hkv][D] and scales [blocks][Hkv],
    in place.  Returns the places whose values are defined afterwards as a mask."""
    defined = np.ones(len(codes), bool)
    for r in range(len(length)):
        T, L = int(prefix[r]), int(length[r])
        old_codes, old_scales = codes.copy(), scales.copy()
        blocks = {}
        for s in range(max(0, T - block), T + L + 1):
            blocks.setdefault(block_of(s, r, page_size, block, table), []).append(s)
        wanted = {block_of(s, r, page_size, block, table) for s in range(T, T + L + 1)}
        for at in wanted:
            src = [s if s < T else T + int(idx[r][s - T]) for s in blocks[at]]
            of = np.array([old_scales[block_of(s, r, page_size, block, table)] for s in src])
            new = of.max(axis=0)
            scales[at] = new
            per = -(-page_size // block)
            first = at // per * page_size + at % per * block
            mine = np.arange(first, min(first + block, (at // per + 1) * page_size))
            kept = [place_of(s, r, page_size, table) for s in blocks[at]]
            defined[np.setdiff1d(mine, kept)] = False
            for s, c, b in zip(kept, src, of):
                v = VALUES[old_codes[place_of(c, r, page_size, table)]]
                codes[s] = encode(v * 2.0 ** (b.astype(float) - new)[:, None])
    return defined
