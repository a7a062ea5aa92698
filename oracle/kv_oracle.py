"""Oracles of the operators around a round.  TEST INFRASTRUCTURE ONLY.

Plain float64 restatements, request by request and row by row, of what
``include/pctree.h`` says of ``pctree_kv_append``, ``pctree_paged_attention``
and ``pctree_sample``.  They share no code with the CUDA library.
"""
from __future__ import annotations

import numpy as np


def place_of(slot, r, page_size, page_table):
    """Place of slot ``slot`` of request r in the cache's [n_pages * page_size]
    places (page_table None: its only page is page r)."""
    page = r if page_table is None else int(page_table[r][slot // page_size])
    return page * page_size + slot % page_size


def norm_rotate(x, weight, position, inv_freq, interleaved, eps, rope_scale=1.0):
    """One head row in float64: norm (weight not None), then rotation of its
    first 2 * len(inv_freq) dims.  Returns the row and, for tolerances, the sum
    of magnitudes that each output adds up."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean() + eps) * np.asarray(weight, np.float64)
    y, size = x.copy(), np.abs(x)
    half = len(inv_freq)
    if half:
        a = np.arange(half) * (2 if interleaved else 1)
        b = a + (1 if interleaved else half)
        t = float(position) * np.asarray(inv_freq, np.float64)
        c, s = np.cos(t) * rope_scale, np.sin(t) * rope_scale
        y[a] = x[a] * c - x[b] * s
        y[b] = x[b] * c + x[a] * s
        size[a] = size[b] = (np.abs(x[a]) + np.abs(x[b])) * abs(rope_scale)
    return y, size


def paged_attention(q, K, V, row_start, n_rows, prefix_len, page_size, page_table, scale):
    """q [rows][Hq][D], K / V [places][Hkv][D] float64.  Returns out (NaN in
    rows of no request) and, for tolerances, sum_s p_s |v_s| beside it."""
    rows, Hq, D = q.shape
    G = Hq // K.shape[1]
    out = np.full((rows, Hq, D), np.nan)
    size = np.zeros((rows, Hq, D))
    for r in range(len(n_rows)):
        T, n, a = int(prefix_len[r]), int(n_rows[r]), int(row_start[r])
        at = np.array([place_of(s, r, page_size, page_table) for s in range(T + n)], np.int64)
        for j in range(n):
            see = at[:T + j + 1]
            for h in range(Hq):
                s = scale * (K[see, h // G] @ q[a + j, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[a + j, h] = p @ V[see, h // G]
                size[a + j, h] = p @ np.abs(V[see, h // G])
    return out, size


def sample_row(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The token of one row of logits (float64 values of the given type)."""
    z = np.asarray(z, np.float64)
    V = len(z)
    order = np.lexsort((np.arange(V), -z))           # (z desc, index asc)
    if temperature == 0:
        return int(order[0])
    if 0 < top_k < V:
        order = order[:top_k]
    with np.errstate(invalid="ignore"):
        w = np.exp((z[order] - z[order[0]]) / float(temperature))
    if top_p < 1:
        cum = np.cumsum(w)
        m = 1 + int(np.searchsorted(cum, float(top_p) * cum[-1], side="left"))
        order, w = order[:m], w[:m]
    some = w >= float(min_p)
    order, w = order[some], w[some]
    by = np.argsort(order)
    cum = np.cumsum(w[by])
    return int(order[by][np.searchsorted(cum, float(u) * cum[-1], side="right")])
