"""The paged KV cache in plain form: numpy, 64-bit floats, one row at a time.  Defines what the HIP kernels of
include/csd.h's csd_paged_* calls compute; shares no code with them.  Pools hold values (not codes) as float64."""
from __future__ import annotations

import numpy as np


def e4m3_round(y):
    """Nearest e4m3 value, ties to even (the sign kept; |y| <= 448 by the caller's scale).  NaN and infinities give NaN."""
    y = np.asarray(y, dtype=np.float64)
    finite = np.isfinite(y)
    a = np.where(finite, np.abs(y), 1.0)
    e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6)
    step = np.exp2(e - 3)
    r = np.rint(a / step) * step
    return np.where(finite, np.copysign(r, y), np.nan)


def scale_byte(x):
    """e + 127 of the rows x [..., D]: the smallest e >= -126 with max |x| <= 448 * 2^e (entries that are not finite do not count)."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.ceil(np.log2(np.where(a > 0, a, 1.0) / 448.0))
    e = np.where(448.0 * np.exp2(e - 1) >= a, e - 1, np.where(448.0 * np.exp2(e) < a, e + 1, e))     # log2 may be a hair off
    return np.where(a > 0, np.maximum(e, -126), -126).astype(np.int64) + 127


def quantise(x):
    """(values the codes stand for, scale bytes) of rows x [..., D]; with the largest scale, 2^120, codes end at 240 (256 would stand
    for 2^128, beyond fp32)."""
    s = scale_byte(x)
    p = np.exp2(s.astype(np.float64) - 127)[..., None]
    y = e4m3_round(x / p)
    return np.where((s == 247)[..., None] & (np.abs(y) > 240), np.copysign(240, y), y) * p, s


def places(row_start, pos, table, page_rows, n_pages, rows):
    """[(row, sequence, position, page or -1, slot)] of every row that belongs to a sequence."""
    out = []
    for b in range(len(pos)):
        for r in range(int(row_start[b]), min(int(row_start[b + 1]), rows)):
            at = int(pos[b]) + r - int(row_start[b])
            i = at // page_rows
            page = int(table[b][i]) if i < table.shape[1] else -1
            out.append((r, b, at, page if 0 <= page < n_pages else -1, at % page_rows))
    return out


def write(pool, rows, where):
    """pool [pages][heads][slots][D] (changed in place) <- rows [n][heads][D]."""
    for r, _, _, page, slot in where:
        if page >= 0:
            pool[page, :, slot] = rows[r]


def read(pool, where, n):
    out = np.zeros((n,) + (pool.shape[1], pool.shape[3]))
    for r, _, _, page, slot in where:
        if page >= 0:
            out[r] = pool[page, :, slot]
    return out


def ancestors(parent):
    """Rows above and including each row of a block."""
    out = []
    for i in range(len(parent)):
        seen, r = {i}, i
        while r > 0:
            p = int(parent[r])
            r = p if 0 <= p < r else 0
            seen.add(r)
        out.append(seen)
    return out


def attention(k, v, table, row_start, cache_len, q, scale, parent=None, out=None):
    """q [rows][heads][D] -> out (given: rows of no sequence keep what it holds)."""
    n_pages, kv_heads, page_rows, _ = k.shape
    rows, heads, d = q.shape
    out = np.zeros((rows, heads, d)) if out is None else np.array(out, dtype=np.float64)
    group = heads // kv_heads
    for b in range(len(cache_len)):
        s, t = int(row_start[b]), int(cache_len[b])
        m = int(row_start[b + 1]) - s
        above = ancestors(parent[s:s + m]) if parent is not None else None
        at = [(p, int(table[b][p // page_rows])) for p in range(min(t + m, table.shape[1] * page_rows))]
        at = [(p, page) for p, page in at if 0 <= page < n_pages]
        pos = np.array([p for p, _ in at], dtype=np.int64)
        page = np.array([g for _, g in at], dtype=np.int64)
        for i in range(m):
            if above is None:
                sees = pos <= t + i
            else:
                sees = np.array([p < t or (p - t) in above[i] for p in pos], dtype=bool)
            if not sees.any():
                out[s + i] = 0
                continue
            kk, vv = k[page[sees], :, pos[sees] % page_rows], v[page[sees], :, pos[sees] % page_rows]    # [n][kv][D]
            for h in range(heads):
                x = scale * (kk[:, h // group] @ q[s + i, h])
                w = np.exp(x - x.max())
                out[s + i, h] = (w / w.sum()) @ vv[:, h // group]
    return out


def commit(pool, table, cache_len, path, n_accepted):
    """pool [layers][pages][heads][slots][D], changed in place."""
    page_rows, n_pages, m = pool.shape[3], pool.shape[1], path.shape[1]

    def place(b, pos):
        i = pos // page_rows
        page = int(table[b][i]) if i < table.shape[1] else -1
        return (page if 0 <= page < n_pages else -1), pos % page_rows

    for b in range(len(cache_len)):
        prev = 0
        for j in range(min(max(int(n_accepted[b]), 0), m - 1)):
            src = int(path[b][j])
            if src <= prev or src < j + 1 or src >= m:
                break
            prev = src
            (sp, ss), (dp, ds) = place(b, int(cache_len[b]) + src), place(b, int(cache_len[b]) + 1 + j)
            if sp >= 0 and dp >= 0:
                pool[:, dp, :, ds] = pool[:, sp, :, ss]
