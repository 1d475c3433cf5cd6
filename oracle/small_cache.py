"""fp64 CPU oracle for 8-bit pages, attention weights and eviction.  TEST INFRASTRUCTURE ONLY, like
recache_oracle.py beside it: plain definitions in numpy float64, nothing from the package.

Pins: tests/test_small_cache_oracle.py (the e4m3 values against torch's own 8-bit type and against the 256 values
enumerated from the format, the scale against a search over exponents, eviction against a sort in plain Python).
"""
from __future__ import annotations

import math

import numpy as np

from .recache_oracle import rope, round_storage

F64 = np.float64
E4M3_MAX = 448.0


def round_e4m3(x):
    """Nearest e4m3 value (4 exponent bits with bias 7, 3 mantissa bits, no infinity), ties to the even last bit;
    |x| <= 448 is the caller's to see to.  NaN and infinities become NaN."""
    x = np.asarray(x, F64)
    fine = np.isfinite(x)
    a = np.where(fine, np.abs(x), 0.0)
    _, e = np.frexp(np.maximum(a, 2.0 ** -6))           # a < 2^e; below 2^-6 the spacing stays 2^-9
    step = np.ldexp(1.0, e - 4)
    return np.where(fine, np.copysign(np.rint(a / step) * step, x), np.nan)


def page_scale(rows) -> float:
    """2^e, e the least integer >= -126 with max|finite x| <= 448 * 2^e; 1 where nothing is above 0."""
    rows = np.asarray(rows, F64)
    a = np.abs(rows[np.isfinite(rows)])
    top = a.max() if a.size else 0.0
    if top == 0.0:
        return 1.0
    e = -126
    while top > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def pack_page(rows):
    """(8-bit values of the rows of one page, scale)."""
    s = page_scale(rows)
    return round_e4m3(np.asarray(rows, F64) / s), s


def rows_of(table, n, page_tokens):
    idx = np.arange(n)
    return table[idx // page_tokens], idx % page_tokens


def attend_decode(q, q_pos, first, k_pages, v_pages, res_table, res_len, hist_table, hist_len, theta, page_tokens, storage=None):
    """One token per sequence over a first part and a history, one softmax.  first: None (the first part's pages are k_pages /
    v_pages) or (k8, v8, k_scale, v_scale) as fp64 values.  Returns (o [B,Hq,d], probability of every row summed over the
    group's heads, as one array per item: first part, then history)."""
    q = np.asarray(q, F64)
    b, hq, d = q.shape
    g = len(res_len) // b
    s = hq // g
    qh = round_storage(rope(q, np.asarray(q_pos), theta), storage)
    o, got = np.zeros_like(q), []
    for it in range(b * g):
        i, kg = divmod(it, g)
        pr, sr = rows_of(res_table[it], int(res_len[it]), page_tokens)
        ph, sh = rows_of(hist_table[it], int(hist_len[it]), page_tokens)
        if first is None:
            kf, vf = k_pages[pr, sr], v_pages[pr, sr]
        else:
            k8, v8, ks, vs = first
            kf, vf = k8[pr, sr] * ks[pr][:, None], v8[pr, sr] * vs[pr][:, None]
        keys = np.concatenate([kf.reshape(-1, d), k_pages[ph, sh].reshape(-1, d)]).astype(F64)
        vals = np.concatenate([vf.reshape(-1, d), v_pages[ph, sh].reshape(-1, d)]).astype(F64)
        sc = qh[i, kg * s:(kg + 1) * s] @ keys.T / math.sqrt(d)
        p = np.exp(sc - sc.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        o[i, kg * s:(kg + 1) * s] = p @ vals
        got.append(p.sum(axis=0))
    return o, got


def keep_rows(weights, budget: int, n_recent: int):
    """Old indices, ascending, of the rows an item of these weights keeps."""
    n = len(weights)
    if n <= budget:
        return list(range(n))
    last = list(range(n - n_recent, n))
    heavy = sorted(range(n - n_recent), key=lambda i: (math.isnan(weights[i]), -weights[i] if not math.isnan(weights[i]) else 0.0, i))
    return sorted(heavy[:budget - n_recent]) + last
