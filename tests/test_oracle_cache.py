"""Pins of the cache oracle: the formats' values from their definitions, rounding by hand, and the operators on cases small
enough to follow."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as orc


def test_e4m3_values_and_rounding():
    v = orc.decode(np.arange(256), orc.E4M3)
    assert v[0x38] == 1.0 and v[0x7e] == 448.0 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0xb8] == -1.0
    assert math.isnan(v[0x7f]) and math.isnan(v[0xff])
    every = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    np.testing.assert_array_equal(orc.encode(orc.decode(every, orc.E4M3), orc.E4M3), every)
    # ties to the even code: 1 + 1/16 lies between 1 (0x38) and 1.125 (0x39), 1 + 3/16 between 0x39 and 0x3a
    assert orc.encode([1 + 1 / 16, 1 + 3 / 16, 1 + 1 / 16 + 1e-9, 2.0 ** -10, 1.5 * 2.0 ** -9, 1e-9], orc.E4M3).tolist() == [
        0x38, 0x3a, 0x39, 0x00, 0x02, 0x00]


def test_int8_values_and_rounding():
    assert orc.decode([0, 1, 127, 128, 129, 255], orc.INT8).tolist() == [0, 1, 127, -128, -127, -1]
    assert orc.encode([0.5, 1.5, -0.5, -2.5, 126.6], orc.INT8).view(np.int8).tolist() == [0, 2, 0, -2, 127]


@pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8])
def test_scale_is_the_smallest_power_of_two(fmt):
    big = orc.LARGEST[fmt]
    for e in (-100, -3, 0, 5, 100):
        assert orc.page_scale([big * 2.0 ** e], fmt) == 2.0 ** e
        assert orc.page_scale([-big * 2.0 ** e * (1 + 2.0 ** -8)], fmt) == 2.0 ** (e + 1)
        assert orc.page_scale([big * 2.0 ** (e - 1) * (1 + 2.0 ** -8), 0.0], fmt) == 2.0 ** e
    assert orc.page_scale([0.0], fmt) == 2.0 ** -126 and orc.page_scale([1e-40], fmt) == 2.0 ** -126
    assert math.isnan(orc.page_scale([1.0, math.inf], fmt)) and math.isnan(orc.page_scale([math.nan], fmt))


def _small(fmt, lens, block=64, pages=3):
    lens = np.asarray(lens, np.int32)
    n = lens.size * pages
    table = np.arange(n, dtype=np.int32)[::-1].reshape(*lens.shape, pages).copy()
    z = lambda: np.full((n, block, orc.D), 0x7f, np.uint8)
    return orc.CacheState(z(), z(), np.ones(n), np.ones(n), table, lens, fmt)


@pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8])
def test_append_grows_a_scale_and_rounds_again(fmt):
    c = _small(fmt, [[2]])
    k = np.zeros((2, 1, orc.D))
    k[0], k[1] = orc.LARGEST[fmt], 1.0
    orc.append(c, k, k, [0, 2])
    p = c.table[0, 0, 0]
    assert c.k_scale[p] == 1.0
    c.lens[:] = 3
    orc.append(c, 4 * k[:1], k[1:], [0, 1])              # keys four times as large, values within the scale
    assert c.k_scale[p] == 4.0 and c.v_scale[p] == 1.0
    got = c.values("k", 0, 0, 3)[:, 0]
    # 1 / 4: exact in e4m3; a tie between 0 and 4 steps of a quarter in int8, to the even one
    assert got.tolist() == [448.0, 1.0, 4 * 448.0] if fmt == orc.E4M3 else got.tolist() == [128.0, 0.0, 508.0]


def test_attn_one_key_and_none():
    c = _small(orc.E4M3, [[1, 0]])
    x = np.ones((1, 2, orc.D))
    c.lens[:] = 1
    orc.append(c, x, 2 * x, [0, 1])
    c.lens[0, 1] = 0
    q = np.ones((2, 2, orc.D))
    out, lse, w, _, _, _ = orc.attn(c, q, [0, 2], [0, 1], scale=1.0, weight_in=np.zeros((1, 2, c.capacity), np.float32))
    assert (out[1, 0] == 2).all() and lse[0, 1] == 128.0 and lse[0, 0] == -np.inf      # the first of two sees nothing
    assert (out[:, 1] == 0).all() and (lse[1] == -np.inf).all()
    assert w[0, 0, 0] == 1.0 and w.sum() == 1.0


def test_evict_order_and_ties():
    c = _small(orc.INT8, [[8]])
    x = np.arange(8.0)[:, None, None] * np.ones((1, 1, orc.D))
    orc.append(c, x, x, [0, 8])
    to = _small(orc.INT8, [[0]])
    w = np.zeros((1, 1, c.capacity), np.float32)
    w[0, 0, :8] = [0, 5, 1, 1, np.nan, 1, -0.0, 0]
    w_out, kept = orc.evict(c, w, np.array([[5]]), 1, 1, to)
    assert kept[0, 0, :5].tolist() == [0, 1, 2, 4, 7] and to.lens[0, 0] == 5
    assert to.values("k", 0, 0, 5)[:, 0].tolist() == [0, 1, 2, 4, 7] and np.isnan(w_out[0, 0, 3])
    orc.evict(c, w, np.array([[0]]), 6, 6, to)
    assert to.lens[0, 0] == 8


def test_codes_near_the_largest_float_stay_finite():
    top = float(np.float32(3.3895314e38))                # bf16's largest
    for fmt, scale, code in ((orc.E4M3, 2.0 ** 120, 240.0), (orc.INT8, 2.0 ** 122, 63.0)):
        assert orc.page_scale([top], fmt) == scale
        assert orc.decode(orc.codes_of([top, -top], scale, fmt), fmt).tolist() == [code, -code] and code * scale < 2.0 ** 128
