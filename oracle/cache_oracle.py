"""CPU oracle of the 8-bit key/value cache, numpy in 64 bits, written from the definitions in include/shplb.h.

A cache here is a CacheState of numpy arrays laid out like the device's; every function works on copies or changes the
state it is given, as its entry point does.  Plain loops over sequences, heads and pages: test infrastructure only.
"""
from __future__ import annotations

import copy
import math
from dataclasses import dataclass

import numpy as np

E4M3, INT8 = 0, 1
LARGEST = {E4M3: 448.0, INT8: 127.0}
D = 128


def decode(codes, fmt):
    c = np.asarray(codes, np.uint8).astype(np.int64)
    if fmt == INT8:
        return np.where(c > 127, c - 256, c).astype(np.float64)
    e, m = (c >> 3) & 15, c & 7
    mag = np.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9.0)
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c > 127, -mag, mag)


_E4M3_MAGNITUDES = decode(np.arange(127), E4M3)          # ascending, code c at place c


def encode(values, fmt):
    """Codes of values (already divided by the scale), to nearest, ties to the even code."""
    y = np.asarray(values, np.float64)
    if fmt == INT8:
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    mag = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(_E4M3_MAGNITUDES, mag), 1, 126)
    lo = hi - 1
    below, above = mag - _E4M3_MAGNITUDES[lo], _E4M3_MAGNITUDES[hi] - mag
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return (np.where(up, hi, lo) | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def page_scale(values, fmt):
    """Smallest power of two, at least 2^-126, with which the values fit; NaN if one is not finite."""
    v = np.asarray(values, np.float64)
    if v.size and not np.isfinite(v).all():
        return math.nan
    amax = float(np.abs(v).max()) if v.size else 0.0
    e = -126
    if amax > 0:
        m, x = math.frexp(amax / LARGEST[fmt])           # m in [1/2, 1)
        e = max(-126, x - 1 if m == 0.5 else x)
        # the quotient is rounded: settle it on the exact products
        while e > -126 and amax <= LARGEST[fmt] * 2.0 ** (e - 1):
            e -= 1
        while amax > LARGEST[fmt] * 2.0 ** e:
            e += 1
    return 2.0 ** e


def codes_of(values, scale, fmt):
    """Codes of a page's values under its scale; at the largest scale they stay at those whose values are below 2^128."""
    if math.isnan(scale):
        return np.zeros(np.shape(values), np.uint8)
    most = LARGEST[fmt]
    if most * scale >= 2.0 ** 128:
        most = 240.0 if fmt == E4M3 else 63.0
    return encode(np.clip(np.asarray(values) / scale, -most, most), fmt)


@dataclass
class CacheState:
    k_pages: np.ndarray        # uint8 [n_pages, block, 128]
    v_pages: np.ndarray
    k_scale: np.ndarray        # float64 [n_pages]
    v_scale: np.ndarray
    table: np.ndarray          # int32 [n_seq, n_kv_heads, max_pages]
    lens: np.ndarray           # int32 [n_seq, n_kv_heads]
    fmt: int

    @property
    def block(self):
        return self.k_pages.shape[1]

    @property
    def n_pages(self):
        return self.k_pages.shape[0]

    @property
    def capacity(self):
        return self.table.shape[2] * self.block

    def copy(self):
        return copy.deepcopy(self)

    def good(self, s, h):
        return 0 <= self.lens[s, h] <= self.capacity

    def values(self, which, s, h, n):
        """The first n tokens of a head."""
        pages, scale = (self.k_pages, self.k_scale) if which == "k" else (self.v_pages, self.v_scale)
        out = np.full((n, D), np.nan)
        for t0 in range(0, n, self.block):
            p, m = int(self.table[s, h, t0 // self.block]), min(self.block, n - t0)
            if 0 <= p < self.n_pages:
                out[t0:t0 + m] = decode(pages[p, :m], self.fmt) * scale[p]
        return out


def append(c: CacheState, k, v, cu):
    """k, v: float64 [n_tokens, n_kv_heads, 128]."""
    for s in range(c.table.shape[0]):
        n = int(cu[s + 1] - cu[s])
        for h in range(c.table.shape[1]):
            if n == 0 or not c.good(s, h):
                continue
            length = int(c.lens[s, h])
            start = max(length - n, 0)
            first_row = int(cu[s]) + start - (length - n)
            for pages, scale, x in ((c.k_pages, c.k_scale, k), (c.v_pages, c.v_scale, v)):
                for i in range(start // c.block, -(-length // c.block)):
                    p = int(c.table[s, h, i])
                    if not 0 <= p < c.n_pages:
                        continue
                    a, b = max(start, i * c.block), min(length, (i + 1) * c.block)
                    fresh = x[first_row + a - start:first_row + b - start, h]
                    held = a - i * c.block
                    new = page_scale(fresh, c.fmt)
                    if held:
                        old = scale[p]
                        new = math.nan if math.isnan(old) or math.isnan(new) else max(old, new)
                        if new != old:
                            again = decode(pages[p, :held], c.fmt) * old
                            pages[p, :held] = codes_of(again, new, c.fmt)
                    pages[p, held:b - i * c.block] = codes_of(fresh, new, c.fmt)
                    scale[p] = new


def load(c: CacheState, k_out, v_out, cu):
    for s in range(c.table.shape[0]):
        n = int(cu[s + 1] - cu[s])
        for h in range(c.table.shape[1]):
            if n == 0 or not c.good(s, h):
                continue
            length = int(c.lens[s, h])
            m = min(n, length)
            for which, out in (("k", k_out), ("v", v_out)):
                out[int(cu[s + 1]) - m:int(cu[s + 1]), h] = c.values(which, s, h, length)[length - m:]


def attn(c: CacheState, q, cu, kv_of, scale=None, weight_in=None):
    """q: float64 [n_tokens, n_q_heads, 128].  Returns out, lse [n_q_heads, n_tokens], weight (or None), and for tolerances
    `size` (sum of p |v|, like out), `all_v` (sum of |v| over the keys seen, likewise) and `reach` (the largest sum of
    |q k| * scale of any pair)."""
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, size, all_v = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    lse = np.zeros((q.shape[1], q.shape[0]))
    weight = None if weight_in is None else weight_in.astype(np.float64).copy()
    reach = 0.0
    for s in range(c.table.shape[0]):
        r0, n = int(cu[s]), int(cu[s + 1] - cu[s])
        for h in range(c.table.shape[1]):
            heads = [x for x in range(q.shape[1]) if kv_of[x] == h]
            if n == 0 or not heads:
                continue
            if not c.good(s, h):
                out[r0:r0 + n, heads] = np.nan
                lse[heads, r0:r0 + n] = np.nan
                continue
            length = int(c.lens[s, h])
            k, v = c.values("k", s, h, length), c.values("v", s, h, length)
            for j in range(n):
                sees = max(0, length - n + 1 + j)
                for x in heads:
                    if sees == 0:
                        lse[x, r0 + j] = -np.inf
                        continue
                    z = (k[:sees] @ q[r0 + j, x]) * scale
                    if not np.isfinite(z).all():
                        out[r0 + j, x], lse[x, r0 + j] = np.nan, np.nan
                        if weight is not None:
                            weight[s, h, :sees] = np.nan
                        continue
                    reach = max(reach, float((np.abs(k[:sees]) @ np.abs(q[r0 + j, x])).max()) * scale)
                    m = z.max()
                    p = np.exp(z - m)
                    lse[x, r0 + j] = m + math.log(p.sum())
                    p /= p.sum()
                    out[r0 + j, x], size[r0 + j, x] = p @ v[:sees], p @ np.abs(v[:sees])
                    all_v[r0 + j, x] = np.abs(v[:sees]).sum(0)
                    if weight is not None:
                        weight[s, h, :sees] += p
    return out, lse, weight, size, all_v, reach


def evict(c: CacheState, weight, keep, n_sink, n_recent, to: CacheState):
    """Fills `to` and returns weights and former positions of the tokens that stay, 0 behind them."""
    w_out = np.zeros(to.table.shape[:2] + (to.capacity,), np.float32)
    kept = np.zeros(w_out.shape, np.int32)
    for s in range(c.table.shape[0]):
        for h in range(c.table.shape[1]):
            if not c.good(s, h):
                to.lens[s, h] = -1
                continue
            length = int(c.lens[s, h])
            n = min(length, to.capacity, max(int(keep[s, h]), n_sink + n_recent))
            sink = min(n_sink, n)
            recent = min(n_recent, n - sink)
            w = weight[s, h, :length].astype(np.float64)
            order = np.where(np.isnan(w), np.inf, w)
            nan_first = np.where(np.isnan(w), 0, 1)
            middle = np.arange(sink, length - recent)
            middle = middle[np.lexsort((middle, -order[middle], nan_first[middle]))][:n - sink - recent]
            at = np.sort(np.concatenate([np.arange(sink), middle, np.arange(length - recent, length)]))
            assert at.size == n
            to.lens[s, h] = n
            kept[s, h, :n], w_out[s, h, :n] = at, weight[s, h, at]
            for which, pages, scale in (("k", to.k_pages, to.k_scale), ("v", to.v_pages, to.v_scale)):
                value = c.values(which, s, h, length)[at]
                for i in range(-(-n // to.block)):
                    p = int(to.table[s, h, i])
                    if not 0 <= p < to.n_pages:
                        continue
                    x = value[i * to.block:(i + 1) * to.block]
                    scale[p] = page_scale(x, c.fmt)
                    pages[p, :x.shape[0]] = codes_of(x, scale[p], c.fmt)
    return w_out, kept
