"""Plain forms of cross attention, verification of drafted tokens and the upkeep of pages, for the tests: float64 or whole numbers on the
CPU, one sequence at a time, written from the definitions (include/quoka.h)."""
from __future__ import annotations

import numpy as np


def cross(q, k, v):
    """q [n_Q, n, d]; k, v [T, n_KV, d] -> out, lse, and P |V| of every element (what relative errors of the probabilities are multiplied
    with)."""
    n_q, n, d = q.shape
    out, weight, lse = np.zeros((n_q, n, d)), np.zeros((n_q, n, d)), np.full((n_q, n), -np.inf)
    if len(k) == 0:
        return out, lse, weight
    for h in range(n_q):
        kv = h // (n_q // k.shape[1])
        z = q[h] @ k[:, kv].T / np.sqrt(d)
        top = z.max(axis=1, keepdims=True, initial=-np.inf)
        p = np.exp(z - top)
        total = p.sum(axis=1, keepdims=True)
        lse[h] = (top + np.log(total))[:, 0]
        p /= total
        out[h], weight[h] = p @ v[:, kv], p @ np.abs(v[:, kv])
    return out, lse, weight


def verify(p, q, tokens, uniform, n):
    """p [n_draft + 1, V], q [n_draft, V] or None, one sequence -> accepted tokens and the row of tokens that comes out."""
    p = np.asarray(p, dtype=np.float64)
    V = p.shape[1]
    u = np.asarray(uniform, dtype=np.float64)
    out = np.full(len(p), -1, dtype=np.int64)
    positive = lambda w: np.where((w > 0) & (w < np.inf), w, 0.0)  # noqa: E731  (NaN compares false)
    a = 0
    while a < n:
        x = int(tokens[a])
        drawn = 1.0 if q is None or not 0 <= x < V else float(q[a][x])
        if not 0 <= x < V or not (float(u[a]) * drawn < p[a][x] and 0 < p[a][x] < np.inf and np.isfinite(drawn)):
            break
        out[a] = x
        a += 1
    w = positive(p[a])
    if a < n:
        if q is None:
            off = np.zeros(V)
            if 0 <= int(tokens[a]) < V:
                off[int(tokens[a])] = 1.0
        else:
            off = np.asarray(q[a], dtype=np.float64)
        with np.errstate(invalid="ignore"):
            left = positive(p[a] - off)
        w = left if left.sum() > 0 else w
    if w.sum() > 0:
        r = u[-1]
        r = 0.0 if not r > 0 else min(r, 1.0 - 2.0 ** -24)
        line = np.cumsum(w)
        out[a] = np.flatnonzero((line > r * line[-1]) & (w > 0))[0]
    return a, out


class Book:
    """Lists of the pages that each sequence holds, over one count of holders."""

    def __init__(self, ref, page_len, batch, max_pages):
        self.ref, self.page_len, self.max_pages = ref, page_len, max_pages
        self.rows = [[] for _ in range(batch)]

    def _take(self, wants):
        """wants: (row, how many more).  -> pages lacking"""
        free = iter([i for i, r in enumerate(self.ref) if r <= 0])
        lacking = 0
        for row, n in wants:
            for _ in range(n):
                page = next(free, None)
                if page is None:
                    lacking += 1
                else:
                    self.ref[page] = 1
                    row.append(page)
        return lacking

    def resize(self, lens):
        n = [min(-(-max(t, 0) // self.page_len), self.max_pages) for t in lens]
        for row, k in zip(self.rows, n):
            for page in row[k:]:
                self.ref[page] -= 1
            del row[k:]
        return self._take([(row, k - len(row)) for row, k in zip(self.rows, n)])

    def fork(self, source, parents, lens):
        """-> first, lens of the children, pages lacking"""
        P = self.page_len
        for row in self.rows:
            for page in row:
                self.ref[page] -= 1
            row.clear()
        n = []
        for row, p in zip(self.rows, parents):
            t = 0
            if 0 <= p < len(source.rows):
                t = min(max(lens[p], 0), min(len(source.rows[p]), self.max_pages) * P)
                for page in source.rows[p][:t // P]:
                    self.ref[page] += 1
                    row.append(page)
            n.append(t)
        first = [t // P * P for t in n]
        lacking = self._take([(row, 1 if t % P else 0) for row, t in zip(self.rows, n)])
        return first, [t if len(row) * P >= t else f for row, t, f in zip(self.rows, n, first)], lacking

    def table(self):
        return np.array([row + [-1] * (self.max_pages - len(row)) for row in self.rows])
