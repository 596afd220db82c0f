"""fp64 CPU oracle for rotary embedding with several axes, the paged key/value cache and the attention over it (test infrastructure).

THIS IS TEST INFRASTRUCTURE: only the tests may import it; the GPU library never does and shares no code with it.

Rotation: as in oracle/rope.py, with a position per axis and token and an axis per pair of columns:
    phi_i = p_{a(i)} base^(-2i/d),  y_i = x_i cos phi_i - x_{i+d/2} sin phi_i,  y_{i+d/2} = x_{i+d/2} cos phi_i + x_i sin phi_i.

Cache: pages [num_pages, heads, page_size, row]; row r of a sequence that brings n rows and has kv tokens cached with them sits at
position kv - n + r; position p lies in slot p % page_size of page table[s, p // page_size].

8-bit rows: e = the smallest integer >= -100 with max |x| <= 448 * 2^e, numbers x / 2^e rounded to e4m3 (sign, 4 exponent bits
with bias 7, 3 mantissa bits; no infinities; 0x7f and 0xff are NaN) to nearest, ties to even.

Attention: the row at position p attends to the keys at positions 0 .. p:
    S_j = scale <q, k_j>,  LSE = ln sum_j exp(S_j),  O = sum_j exp(S_j - LSE) v_j;  no key: O = 0, LSE = -inf.
"""
from __future__ import annotations

import numpy as np


def turn_axes(x, positions, pair_axis, base=10000.0, inverse=False):
    """x [T, H, d], positions [axes, T], pair_axis [d/2]."""
    x = np.asarray(x, dtype=np.float64)
    half = x.shape[-1] // 2
    theta = np.float64(base) ** (-2.0 * np.arange(half) / x.shape[-1])
    phi = np.asarray(positions, dtype=np.float64)[np.asarray(pair_axis)].T * theta       # [T, half]
    c, s = np.cos(phi)[:, None], (-1.0 if inverse else 1.0) * np.sin(phi)[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)


def _e4m3_values():
    out = np.empty(256)
    for b in range(256):
        sign, e, m = (-1.0 if b & 128 else 1.0), (b >> 3) & 15, b & 7
        out[b] = np.nan if b & 127 == 127 else sign * ((8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9)
    return out


E4M3 = _e4m3_values()


def exponent_of(row_max):
    """The smallest e >= -100 with row_max <= 448 * 2^e."""
    e = -100
    while row_max > 448.0 * 2.0 ** e:
        e += 1
    return e


def to_e4m3(x):
    """The codes of x rounded to nearest even; |x| <= 448 or NaN."""
    x = np.asarray(x, dtype=np.float64)
    grid = E4M3[:127]                                   # codes 0 .. 126: 0 .. 448, ascending
    a = np.abs(np.where(np.isnan(x), 0.0, x))
    hi = np.searchsorted(grid, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    mid = (grid[lo] + grid[hi]) / 2
    code = np.where(a > mid, hi, np.where(a < mid, lo, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a == grid[hi], hi, code)
    return np.where(np.isnan(x), 127, code + np.where(np.signbit(x) & ~np.isnan(x), 128, 0)).astype(np.uint8)


def quantise(rows):
    """rows [..., d] -> (codes, scale bytes [...])."""
    rows = np.asarray(rows, dtype=np.float64)
    finite = np.isfinite(rows)
    top = np.where(finite, np.abs(rows), 0.0).max(axis=-1)
    e = np.vectorize(exponent_of, otypes=[np.int64])(top)
    return to_e4m3(np.where(finite, rows, np.nan) * 2.0 ** -e[..., None].astype(np.float64)), (e + 127).astype(np.uint8)


def dequantise(codes, scale):
    return E4M3[codes] * 2.0 ** (scale.astype(np.float64)[..., None] - 127.0)


def places(cu_rows, kv_lens, page_table, page_size, num_pages):
    """For every row of a sequence: (row, sequence, position, page, slot); page -1: none that exists, position < 0: no place."""
    out = []
    for s in range(len(kv_lens)):
        n = cu_rows[s + 1] - cu_rows[s]
        for r in range(n):
            p = kv_lens[s] - n + r
            page = -1
            if p >= 0:
                page = int(page_table[s][p // page_size])
                page = page if 0 <= page < num_pages else -1
            out.append((cu_rows[s] + r, s, p, page, p % page_size if p >= 0 else 0))
    return out


def gather(pool, page_table, kv, page_size):
    """pool [num_pages, H, page_size, d] values -> one sequence's [kv, H, d]; NaN where the page does not exist."""
    out = np.full((kv, pool.shape[1], pool.shape[3]), np.nan)
    for p in range(kv):
        page = int(page_table[p // page_size])
        if 0 <= page < pool.shape[0]:
            out[p] = pool[page, :, p % page_size]
    return out


def attention(q, k_pool, v_pool, cu_rows, kv_lens, page_table, page_size, scale):
    """q [T, Hq, d]; returns O [T, Hq, d] and LSE [Hq, T]; rows that belong to no sequence: NaN.  A masked key takes no part, whatever
    its value: its weight is not 0 times it."""
    T, hq, d = q.shape
    group = hq // k_pool.shape[1]
    o, lse = np.full((T, hq, d), np.nan), np.full((hq, T), np.nan)
    for s, kv in enumerate(kv_lens):
        n = cu_rows[s + 1] - cu_rows[s]
        k, v = gather(k_pool, page_table[s], kv, page_size), gather(v_pool, page_table[s], kv, page_size)
        for r in range(n):
            seen = max(kv - n + r + 1, 0)
            row = cu_rows[s] + r
            for h in range(hq):
                if seen == 0:
                    o[row, h], lse[h, row] = 0.0, -np.inf
                    continue
                x = scale * (k[:seen, h // group] @ q[row, h])
                top = x.max()
                w = np.exp(x - top)
                o[row, h], lse[h, row] = (w / w.sum()) @ v[:seen, h // group], top + np.log(w.sum())
    return o, lse
