"""Test-side plumbing of the 8-bit cache: the same cache as numpy arrays (the oracle's) and as device buffers."""
from __future__ import annotations

import numpy as np
import torch

import paper_2603_10353_amd as S
from oracle import cache_oracle as orc

DEV = "cuda:0"
D = 128


def bf16(x):
    """float array -> (bf16 tensor on the CPU, its values in 64 bits)."""
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16)
    return t, t.to(torch.float64).numpy()


def state(rng, lens, block, fmt, spare=1, extra_pages=2, max_pages=None):
    """A cache whose pages hold bytes of all kinds (NaN codes among them); pages in no order, unused entries -1."""
    lens = np.asarray(lens, np.int32)
    nb = -(-np.maximum(lens, 0) // block)
    width = int(nb.max()) + spare if max_pages is None else max_pages
    need = np.arange(width) < np.minimum(nb + spare, width)[..., None]
    n = int(need.sum())
    table = np.full(need.shape, -1, np.int32)
    table[need] = rng.permutation(n + extra_pages)[:n]
    n += extra_pages
    pages = lambda: rng.integers(0, 256, size=(n, block, D)).astype(np.uint8)
    scale = lambda: np.where(rng.random(n) < 0.5, 1.0, 0.25)
    return orc.CacheState(pages(), pages(), scale(), scale(), table, lens.copy(), fmt)


def filled(rng, lens, block, fmt, size=1.0, **kw):
    """... and with tokens of noise in it, some pages larger than others."""
    c = state(rng, lens, block, fmt, **kw)
    n = np.maximum(c.lens, 0).max(1)
    cu = np.concatenate([[0], np.cumsum(n)])
    shape = (int(cu[-1]), c.table.shape[1], D)
    x = lambda: bf16(size * rng.standard_normal(shape) * np.exp(rng.normal(size=(shape[0], 1, 1)) * 0.5))[1]
    orc.append(c, x(), x(), cu)
    return c


class Device:
    """A CacheState's buffers on the device and its handle."""

    def __init__(self, c: orc.CacheState, device=DEV):
        up = lambda a, t=None: torch.from_numpy(np.ascontiguousarray(a if t is None else a.astype(t))).to(device)
        self.fmt, self.block = c.fmt, c.block
        self.k_pages, self.v_pages = up(c.k_pages), up(c.v_pages)
        self.k_scale, self.v_scale = up(c.k_scale, np.float32), up(c.v_scale, np.float32)
        self.table, self.lens = up(c.table), up(c.lens)
        self.n_seq, self.n_kv_heads, self.max_pages = c.table.shape
        self.cache = S.Cache(self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.table, self.lens, self.n_seq,
                             self.n_kv_heads, c.block, self.max_pages, c.n_pages,
                             S.SHPLB_CACHE_E4M3 if c.fmt == orc.E4M3 else S.SHPLB_CACHE_INT8)

    def check_same(self, c: orc.CacheState):
        """Every byte of the pools and every scale is the oracle's."""
        for mine, theirs in ((self.k_pages, c.k_pages), (self.v_pages, c.v_pages)):
            np.testing.assert_array_equal(mine.cpu().numpy(), theirs)
        for mine, theirs in ((self.k_scale, c.k_scale), (self.v_scale, c.v_scale)):
            np.testing.assert_array_equal(mine.cpu().numpy(), theirs.astype(np.float32))
        np.testing.assert_array_equal(self.lens.cpu().numpy(), c.lens)


def strided(t, extra):
    """A [T, H, 128] tensor on the device as columns of a wider one (extra more heads), and that one."""
    wide = torch.full((t.shape[0], t.shape[1] + extra, D), 7.0, dtype=t.dtype, device=DEV)
    wide[:, extra // 2:extra // 2 + t.shape[1]] = t.to(DEV)
    return wide[:, extra // 2:extra // 2 + t.shape[1]], wide


def step_of(dev: Device, new, hq, ragged, **kw):
    """The step with `new` tokens per sequence (and the device's cu_tokens, kept alive by it)."""
    new = np.asarray(new)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    if not ragged:
        assert len(set(new.tolist())) == 1
        return S.Step(dev.n_seq, hq, dev.n_kv_heads, int(cu[-1]), int(new[0]), None, **kw), cu
    return S.Step(dev.n_seq, hq, dev.n_kv_heads, int(cu[-1]) + kw.pop("behind", 0), int(new.max()), torch.from_numpy(cu).to(DEV), **kw), cu


def attn_workspace(dev, step):
    return torch.empty(S.shplb_cache_attn_workspace_bytes(dev.cache, step), dtype=torch.uint8, device=DEV).fill_(0xff)


def check_attn(c, got_out, got_lse, q, cu, kv_of, scale=None, got_weight=None, weight_in=None, rows=None):
    """Against the oracle.  Tolerances, each a sum of what rounds: a score is a sum of 128 exact products in fp32, in an order and
    with intermediate roundings of the matrix pipe's own (two halves of a step each): 2 * 130 * 2^-24 of the sum of their magnitudes,
    and as much as 2^-23 of itself for each of three multiplications; a probability moves by as much as its score and the
    denominator's logarithm do, 2^-22 for each exponential, n additions of the denominator taken 64 apart; fp16
    probabilities 2^-11, the result bf16 2^-8.  Probabilities are held at 2^7 times their size against a reference that is never above the largest one, and
    fp16's steps end at 2^-24: half a step is 2^-25 * 2^-7 = 2^-32 of the reference, at most 2^-32 of |v| for each key."""
    out, lse, weight, size, all_v, reach = orc.attn(c, q, cu, kv_of, scale, weight_in)
    n = max(1, int(np.maximum(c.lens, 0).max()))
    dz = reach * (2 * 130 * 2.0 ** -24 + 3 * 2.0 ** -23)
    dp = 2 * dz + 2.0 ** -21 + (n / 64 + 80) * 2.0 ** -24
    there = slice(0, int(cu[-1]))
    tol = 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + dp) * size * (1 + 2.0 ** -8) + 2.0 ** -32 * all_v + 1e-30
    diff = np.abs(got_out[there] - out[there])
    assert (np.isnan(got_out[there]) == np.isnan(out[there])).all()
    worst = np.nanmax(np.where(np.isnan(diff), 0, diff / tol[there]), initial=0.0)
    assert worst <= 1.0, "output off by %.3g of the tolerance" % worst
    if got_lse is not None:
        a, b = got_lse[:, there], lse[:, there]
        assert (np.isnan(a) == np.isnan(b)).all() and (np.isneginf(a) == np.isneginf(b)).all()
        fine = np.isfinite(b)
        assert (np.abs(a[fine] - b[fine]) <= dz + dp + 2.0 ** -22 * (np.abs(b[fine]) + 16)).all()
    if got_weight is not None:
        total = max(1, int(np.diff(cu).max())) * len(kv_of)
        for s in range(c.table.shape[0]):
            for h in range(c.table.shape[1]):
                m = int(c.lens[s, h]) if c.good(s, h) else 0
                a, b = got_weight[s, h, :m], weight[s, h, :m]
                assert (np.isnan(a) == np.isnan(b)).all()
                fine = ~np.isnan(b)
                assert (np.abs(a - b)[fine] <= (dp + total * 2.0 ** -23) * np.abs(b[fine]) + 1e-30).all()
    return worst
