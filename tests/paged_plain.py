"""Caches in pages for the tests: the 8-bit format, pools with their page tables, and attention, all in float64 on the CPU and
written from the definitions (include/quoka.h)."""
from __future__ import annotations

import numpy as np
import torch

from gen.workloads import bf16_round


def quantise(rows):
    """rows [..., d] (values of bfloat16 or float32) -> (what the elements stand for without their row's power of two, biased
    exponents)."""
    x = np.asarray(rows, dtype=np.float64)
    top = np.abs(x).max(axis=-1)
    m, e2 = np.frexp(top)                           # top = m * 2^e2, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = np.where(top == 0, -126, np.maximum(e2 - 9 + (m > 0.875), -126))
    y = np.ldexp(x, -e[..., None])
    _, ye = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(ye - 1, -6) - 3)   # three bits behind the leading one; 2^-9 below 2^-6
    return np.rint(y / step) * step, (e + 127).astype(np.int64)


def store(x, dtype):
    return bf16_round(np.asarray(x, dtype=np.float32)) if dtype == "bf16" else np.asarray(x, dtype=np.float32)


TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def to_dev(x, dtype, dev):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dev).to(TORCH[dtype])


class Pool:
    """Pages with rows of every sequence in them (positions 0 .. n - 1 of sequence b: k[b], v[b] [n, n_KV, d]); every other byte
    holds what must never be used."""

    def __init__(self, rng, k, v, n_kv, d, page_len, dtype, fp8, dev="cuda:0", spare=3, table_cols=None, layout="heads", n_pages=None,
                 tail_entries=-1, reserve=None):
        lens = [len(x) for x in k]
        reserve = lens if reserve is None else reserve
        counts = [-(-r // page_len) for r in reserve]
        self.page_len, self.fp8, self.dtype = page_len, fp8, dtype
        cols = max(max(counts), 1) if table_cols is None else table_cols
        n_pages = sum(counts) + spare if n_pages is None else n_pages
        order = rng.permutation(n_pages)
        self.table = np.full((len(k), cols), tail_entries, dtype=np.int64)
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = order[at:at + n]
            at += n
        kt = torch.float8_e4m3fn if fp8 else TORCH[dtype]
        shape = (n_pages, n_kv, page_len, d)
        made = []
        for rows in (k, v):
            if layout == "heads":
                pages = torch.empty(shape, dtype=kt, device=dev)
            else:   # tokens outside heads, and 16 unused elements behind every row
                pages = torch.empty((n_pages, page_len, n_kv, d + 16), dtype=kt, device=dev)[..., :d].permute(0, 2, 1, 3)
            bits = pages.view(torch.uint8) if fp8 else pages
            if fp8:
                bits.fill_(0x7F)   # NaN
                scale = torch.full(shape[:3], 255, dtype=torch.uint8, device=dev)
            else:
                pages.fill_(float("nan"))
                scale = None
            values = []
            for b, x in enumerate(rows):
                x = np.asarray(x, dtype=np.float64).reshape(-1, n_kv, d)
                p = np.arange(len(x))
                page = torch.from_numpy(self.table[b][p // page_len]).to(dev)
                slot = torch.from_numpy(p % page_len).to(dev)
                if len(x) == 0:
                    values.append(x)
                elif fp8:
                    y, e = quantise(x)
                    y8 = torch.from_numpy(y.astype(np.float32)).to(dev).to(torch.float8_e4m3fn)
                    bits[page, :, slot] = y8.view(torch.uint8)
                    scale[page, :, slot] = torch.from_numpy(e).to(dev).to(torch.uint8)
                    values.append(np.ldexp(y, (e - 127)[..., None]))
                else:
                    pages[page, :, slot] = to_dev(x, dtype, dev)
                    values.append(x)
            made.append((pages, scale, values))
        (self.k_pages, self.k_scale, self.k), (self.v_pages, self.v_scale, self.v) = made
        self.dev_table = torch.from_numpy(self.table).to(torch.int32).to(dev)

    def cache(self):
        import paper_2602_08722_amd as pk
        return pk.PagedCache(self.k_pages, self.v_pages, self.dev_table, self.k_scale, self.v_scale)


def attention(q, k, v, n_before, lists=None):
    """q [n_Q, n, d] of one sequence's n tokens; k, v [n_before + n, n_KV, d].  -> out, lse, and P |V| of every element (what
    relative errors of the probabilities are multiplied with), all [n_Q, n, ...] float64."""
    n_q, n, d = q.shape
    n_kv = k.shape[1]
    out = np.zeros((n_q, n, d))
    lse = np.full((n_q, n), -np.inf)
    weight = np.zeros((n_q, n, d))
    if n == 0:
        return out, lse, weight
    hidden = np.triu(np.ones((n, n), dtype=bool), 1)
    for h in range(n_q):
        kv = h // (n_q // n_kv)
        old = np.arange(n_before) if lists is None else np.asarray(lists[kv], dtype=np.int64)
        rows = np.concatenate([old, n_before + np.arange(n)])
        kk, vv = k[rows, kv], v[rows, kv]
        z = q[h] @ kk.T / np.sqrt(d)
        z[:, len(old):][hidden] = -np.inf
        top = z.max(axis=1, keepdims=True)
        p = np.exp(z - top)
        total = p.sum(axis=1, keepdims=True)
        p /= total
        out[h], weight[h] = p @ vv, p @ np.abs(vv)
        lse[h] = (top + np.log(total))[:, 0]
    return out, lse, weight


def attention_spread(q, k, v, n_before, lists=None):
    """As `attention`: sqrt(sum_j P_j^2 V_j^2) of every element, what independent relative errors of the probabilities are multiplied
    with, and the largest magnitude of a visible logit of every row."""
    n_q, n, d = q.shape
    spread, top = np.zeros((n_q, n, d)), np.zeros((n_q, n))
    hidden = np.triu(np.ones((n, n), dtype=bool), 1)
    for h in range(n_q):
        kv = h // (n_q // k.shape[1])
        old = np.arange(n_before) if lists is None else np.asarray(lists[kv], dtype=np.int64)
        rows = np.concatenate([old, n_before + np.arange(n)])
        z = q[h] @ k[rows, kv].T / np.sqrt(d)
        z[:, len(old):][hidden] = -np.inf
        p = np.exp(z - z.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        spread[h] = np.sqrt(p ** 2 @ v[rows, kv] ** 2)
        top[h] = np.abs(np.where(np.isinf(z), 0.0, z)).max(axis=1)
    return spread, top
