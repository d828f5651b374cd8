"""What stands around a review in a serving step, in plain form: numpy, 64-bit floats, one row and one page at a time.  Defines what the HIP kernels of
include/csd.h's csd_pages_*, csd_sample, csd_filter_probs and csd_paged_cross_attention calls compute; shares no code with them."""
from __future__ import annotations

import numpy as np


def weights(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, largest=np.finfo(np.float32).max):
    """(weights of a row by token, slack of every decision): w in 64 bits, 0 for tokens that are left out; slack[v] is how far token v is from being decided
    otherwise, in units of the largest weight (inf where no sum or comparison of weights decides).  largest: the number that infinity counts as."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.float64(largest)))
    n = len(x)
    slack = np.full(n, np.inf)
    m = x.max()
    if m == -np.inf:
        return np.zeros(n), slack
    order = np.lexsort((np.arange(n), -x))                 # by logit, of equal ones the lowest first
    if not temperature > 0:
        w = np.zeros(n)
        w[order[0]] = 1.0
        return w, slack
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(x == m, 0.0, np.where(x == -np.inf, -np.inf, (x - m) / np.float64(temperature)))
    w = np.exp(y)
    if 0 < top_k < n:
        order = order[:top_k]
    if top_p < 1:
        run = np.cumsum(w[order])
        target = max(float(top_p), 0.0) * run[-1]
        before = run - w[order]
        near = np.abs(before - target)
        near[0] = np.inf                                   # the first one stays whatever the sums
        slack[order] = near
        keep = before < target
        keep[0] = True
        order = order[keep]
    least = min(float(min_p), 1.0)
    if least > 0:
        slack = np.minimum(slack, np.where(w == 1.0, np.inf, np.abs(w - least)))
        order = order[w[order] >= least]
    out = np.zeros(n)
    out[order] = w[order]
    return out, slack


def draw(w, u):
    """The lowest token at which the running sum of w passes u times all of it; -1 for a row without weight."""
    run = np.cumsum(w)
    if not run[-1] > 0:
        return -1
    return int(np.searchsorted(run, min(max(float(u), 0.0), 1 - 2.0 ** -24) * run[-1], side="right"))


class Pages:
    """The arrays of csd_pages as lists."""

    def __init__(self, table, held, free, users, page_rows):
        self.table, self.held, self.free, self.users = [list(map(int, r)) for r in table], list(map(int, held)), list(map(int, free)), list(map(int, users))
        self.page_rows, self.n_pages = page_rows, len(self.users)

    def plan(self, cache_len, new_rows, rows):
        width, R = len(self.table[0]), self.page_rows
        row_start, served, n_free, wanted, total = [0], [], len(self.free), 0, 0
        sequence, position, slot = [-1] * rows, [-1] * rows, [-1] * rows
        for b in range(len(self.held)):
            t, n = max(int(cache_len[b]), 0), max(int(new_rows[b]), 0)
            need = max(-(-(t + n) // R) - self.held[b], 0)
            ok = -(-(t + n) // R) <= width
            if ok and n:
                # rows of a page that others use too are not this sequence's to write
                mine = self.table[b][t // R:min(self.held[b], -(-(t + n) // R))]
                ok = not any(0 <= page < self.n_pages and self.users[page] > 1 for page in mine)
            if ok:
                wanted += need
                total += n
                ok = (need == 0 or wanted <= n_free) and (n == 0 or total <= rows)
            if not ok:
                need = n = 0
            served.append(int(ok))
            for _ in range(need):
                page = self.free.pop()
                self.table[b][self.held[b]] = page
                self.users[page] = 1
                self.held[b] += 1
            for i in range(n):
                r = row_start[-1] + i
                page = self.table[b][(t + i) // R]
                sequence[r], position[r], slot[r] = b, t + i, page * R + (t + i) % R if 0 <= page < self.n_pages else -1
            row_start.append(row_start[-1] + n)
        return row_start, sequence, position, slot, served

    def release(self, keep_len):
        back = []
        for b in range(len(self.held)):
            if keep_len[b] < 0:
                continue
            kept = min(-(-int(keep_len[b]) // self.page_rows), self.held[b])
            for i in range(kept, self.held[b]):
                back.append(self.table[b][i])
                self.table[b][i] = -1
            self.held[b] = kept
        back = [p for p in back if 0 <= p < self.n_pages]
        for p in back:
            self.users[p] -= 1
        first = [p for i, p in enumerate(back) if self.users[p] == 0 and p not in back[:i]]
        self.free.extend(reversed(first))

    def share(self, source, length):
        for b in range(len(self.held)):
            s = int(source[b])
            if s < 0 or s >= len(self.held) or s == b or self.held[b] > 0 or source[s] >= 0:
                continue
            n = min(max(int(length[b]), 0) // self.page_rows, self.held[s])
            for i in range(n):
                page = self.table[b][i] = self.table[s][i]
                if 0 <= page < self.n_pages:
                    self.users[page] += 1
            self.held[b] = n


def cross_attention(k, v, table, row_start, enc_len, q, scale, out=None):
    """k, v [pages][kv heads][slots][D], q [rows][heads][D] -> out (given: rows of no sequence keep what it holds)."""
    n_pages, kv_heads, page_rows, _ = k.shape
    rows, heads, d = q.shape
    out = np.zeros((rows, heads, d)) if out is None else np.array(out, dtype=np.float64)
    group = heads // kv_heads
    for b in range(len(enc_len)):
        at = [(int(table[b][p // page_rows]), p % page_rows) for p in range(min(max(int(enc_len[b]), 0), table.shape[1] * page_rows))]
        at = [(page, slot) for page, slot in at if 0 <= page < n_pages]
        page, slot = np.array([a for a, _ in at], dtype=np.int64), np.array([s for _, s in at], dtype=np.int64)
        for r in range(int(row_start[b]), int(row_start[b + 1])):
            if not at:
                out[r] = 0
                continue
            kk, vv = k[page, :, slot], v[page, :, slot]      # [n][kv][D]
            for h in range(heads):
                x = scale * (kk[:, h // group] @ q[r, h])
                w = np.exp(x - x.max())
                out[r, h] = (w / w.sum()) @ vv[:, h // group]
    return out
