"""CPU oracle, in 64 bits, of attention that sees part of a context: a sliding window with first tokens that stay visible, in prefill
and over the 8-bit cache, and sequences that share a prefix in the cache.  Written from the definitions, a query at a time:
position p sees the positions t <= p with t > p - window or t < n_sink; behind a prefix, all of it and the own positions t <= p.
"""
from __future__ import annotations

import math

import numpy as np

from oracle.cache_oracle import decode

D = 128


class Result:
    """Outputs, logarithms of denominators, and for tolerances `size` (sum of p |v|, like out), `all_v` (sum of |v| over the keys seen,
    likewise) and `reach` (the largest sum of |q k| * scale of any pair)."""

    def __init__(self, q):
        self.out, self.size, self.all_v = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
        self.lse = np.full((q.shape[1], q.shape[0]), -np.inf)
        self.reach = 0.0

    def put(self, row, head, q, k, v, scale, only_finite):
        """The query's attention over keys k and values v.  only_finite: products that are no finite numbers make all of it NaN."""
        if len(k) == 0:
            return
        with np.errstate(all="ignore"):
            z = (k @ q) * scale
            if not np.isfinite(z).all() and (only_finite or np.isnan(z).any() or np.isposinf(z).any()):
                self.out[row, head], self.lse[head, row] = np.nan, np.nan
                return
            m = z.max()
            if np.isneginf(m):
                self.out[row, head] = np.nan
                return
            self.reach = max(self.reach, float((np.abs(k[np.isfinite(z)]) @ np.abs(q)).max()) * scale)
            p = np.exp(z - m)
            self.lse[head, row] = m + math.log(p.sum())
            p /= p.sum()
            self.out[row, head], self.size[row, head], self.all_v[row, head] = p @ v, p @ np.abs(v), np.abs(v).sum(0)


def seen(p, n, n_sink, window):
    """The positions below n that position p sees."""
    t = np.arange(max(0, min(n, p + 1)))
    return t[(t > p - window) | (t < n_sink)]


def window_attention(q, k, v, cu, n_sink, window, kv_of, scale=None):
    """q [T, heads, 128], k and v [T, KV heads, 128], float64."""
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    got = Result(q)
    for s in range(len(cu) - 1):
        t0, n = int(cu[s]), int(cu[s + 1] - cu[s])
        for p in range(n):
            at = t0 + seen(p, n, n_sink, window)
            for h in range(q.shape[1]):
                got.put(t0 + p, h, q[t0 + p, h], k[at, kv_of[h]], v[at, kv_of[h]], scale, False)
    return got


def _values_at(c, s, h, at):
    """Keys and values of a head of a cache at these positions; NaN in pages that are not in the pool."""
    at = np.asarray(at, np.int64)
    page = c.table[s, h, at // c.block]
    there = (page >= 0) & (page < c.n_pages)
    page = np.where(there, page, 0)
    got = []
    for pages, scales in ((c.k_pages, c.k_scale), (c.v_pages, c.v_scale)):
        x = decode(pages[page, at % c.block], c.fmt) * scales[page][:, None]
        got.append(np.where(there[:, None], x, np.nan))
    return got


def _rows(q, cu, kv_of, h):
    return [x for x in range(q.shape[1]) if kv_of[x] == h]


def cache_window(c, q, cu, kv_of, n_sink, window, scale=None):
    """q: float64 [tokens, heads, 128], of sequence s the rows cu[s] .. cu[s + 1] - 1, its last ones."""
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    got = Result(q)
    for s in range(c.table.shape[0]):
        r0, n = int(cu[s]), int(cu[s + 1] - cu[s])
        for h in range(c.table.shape[1]):
            heads = _rows(q, cu, kv_of, h)
            for j in range(n):
                if not c.good(s, h):
                    got.out[r0 + j, heads], got.lse[heads, r0 + j] = np.nan, np.nan
                    continue
                length = int(c.lens[s, h])
                k, v = _values_at(c, s, h, seen(length - n + j, length, n_sink, window))
                for x in heads:
                    got.put(r0 + j, x, q[r0 + j, x], k, v, scale, True)
    return got


def cache_shared(prefix, cu_prefix, c, q, cu, kv_of, scale=None):
    """Sequences cu_prefix[g] .. cu_prefix[g + 1] - 1 share prefix g, whose tokens come in front of their own."""
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    got = Result(q)
    for s in range(c.table.shape[0]):
        r0, n = int(cu[s]), int(cu[s + 1] - cu[s])
        of = [g for g in range(len(cu_prefix) - 1) if cu_prefix[g] <= s < cu_prefix[g + 1]]
        for h in range(c.table.shape[1]):
            heads = _rows(q, cu, kv_of, h)
            if not c.good(s, h) or not all(prefix.good(g, h) for g in of):
                got.out[r0:r0 + n, heads] = np.nan
                got.lse[heads, r0:r0 + n] = np.nan
                continue
            front = [_values_at(prefix, g, h, np.arange(int(prefix.lens[g, h]))) for g in of]
            length = int(c.lens[s, h])
            own = _values_at(c, s, h, np.arange(length))
            for j in range(n):
                sees = max(0, length - n + 1 + j)
                k, v = (np.concatenate([*(f[x] for f in front), own[x][:sees]]) for x in (0, 1))
                for x in heads:
                    got.put(r0 + j, x, q[r0 + j, x], k, v, scale, True)
    return got
