"""What the tests of windows and shared prefixes have in common: the comparison with the oracle, caches of many pages."""
from __future__ import annotations

import numpy as np
import torch

import paper_2603_10353_amd as S
from cache_harness import D, Device
from oracle import cache_oracle


def check(want, got_out, got_lse, rows, keys, half_probability, lift=0.0):
    """Against the oracle's Result on these rows.  Tolerances, each a sum of what rounds: a score is a sum of 128 exact products in
    fp32, in an order and with intermediate roundings of the matrix pipe's own (two halves of a step each): 2 * 130 * 2^-24 of the
    sum of their magnitudes, and as much as 2^-23 of itself for each of three multiplications; a probability moves by as much as its
    score and the denominator's logarithm do, 2^-22 for each exponential, the additions of the denominator, `keys` of them at most
    taken 64 apart, and eight times the output is scaled, 2^-22 each; probabilities are rounded before they meet the values, by
    half_probability of themselves or lift of the reference; the result in bf16, 2^-8."""
    dz = want.reach * (2 * 130 * 2.0 ** -24 + 3 * 2.0 ** -23)
    dp = 2 * dz + 2.0 ** -21 + (keys / 64 + 80) * 2.0 ** -24 + 8 * 2.0 ** -22
    out, lse = want.out[rows], want.lse[:, rows]
    a = got_out[rows]
    assert (np.isnan(a) == np.isnan(out)).all(), "NaN where there is none, or none where there is"
    infinite = np.isinf(out)
    assert (a[infinite] == out[infinite]).all()
    fine = np.isfinite(out)
    tol = 2.0 ** -8 * np.abs(out) + (half_probability + dp) * want.size[rows] * (1 + 2.0 ** -8) + lift * want.all_v[rows] + 1e-30
    worst = float((np.abs(a - out)[fine] / tol[fine]).max(initial=0.0))
    assert worst <= 1.0, "output off by %.3g of the tolerance" % worst
    if got_lse is not None:
        b = got_lse[:, rows]
        assert (np.isnan(b) == np.isnan(lse)).all() and (np.isneginf(b) == np.isneginf(lse)).all()
        fine = np.isfinite(lse)
        assert (np.abs(b[fine] - lse[fine]) <= dz + dp + 2.0 ** -22 * (np.abs(lse[fine]) + 16)).all()
    return worst


def in_a_large_pool(c):
    """The CacheState on the device, its pages at the end of a pool of more than 2^32 bytes."""
    behind = -(-2 ** 32 // (c.block * D)) + 3
    dev = Device(c)
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        small = getattr(dev, name)
        large = torch.empty((behind + c.n_pages, *small.shape[1:]), dtype=small.dtype, device=small.device)
        large[behind:] = small
        setattr(dev, name, large)
    dev.table += behind * (dev.table >= 0).int()
    dev.cache = S.Cache(dev.k_pages, dev.v_pages, dev.k_scale, dev.v_scale, dev.table, dev.lens, dev.n_seq, dev.n_kv_heads, c.block,
                        dev.max_pages, behind + c.n_pages, S.SHPLB_CACHE_E4M3 if c.fmt == cache_oracle.E4M3 else S.SHPLB_CACHE_INT8)
    return dev


def far_apart(rng, shape, size, order):
    """Multiples 1 .. 14 of one vector of 2^size and -2^size (for keys: shape (tokens, heads)): products with others of the kind are sums without
    rounding, in the cache's formats, too, and no two of them that differ are closer than a fourteenth."""
    times = rng.integers(1, 15, shape)
    if order == "rising":
        times = np.sort(times, 0)
    return times[..., None] * (1.0 - 2.0 * (np.arange(D) % 3 == 0)) * 2.0 ** size * (-1.0 if order == "below_zero" else 1.0)


def check_far(want, got_out, got_lse, rows, half_probability):
    """Against the oracle's Result where scores are those of far_apart(), times 2^20 and more, so that only the largest ones of a row count, all of them alike:
    what rounds is a probability, the output (2^-8), and, of the largest score, its products with the scales, the logarithm and their sum (2^-22 of it)."""
    out, lse, a, b = want.out[rows], want.lse[:, rows], got_out[rows], got_lse[:, rows]
    assert np.isfinite(a).all() and np.isfinite(b).all()
    assert (np.abs(a - out) <= 2.0 ** -8 * np.abs(out) + half_probability * (1 + 2.0 ** -8) * want.size[rows] + 1e-30).all()
    assert (np.abs(b - lse) <= 2.0 ** -22 * np.abs(lse)).all()
