"""Pins of the oracle of windows and shared prefixes: what is seen, counted by hand, and results that follow from other definitions."""
import numpy as np
import pytest

from oracle import cache_oracle, window_oracle as orc


def test_what_positions_see():
    assert orc.seen(0, 10, 0, 1).tolist() == [0]
    assert orc.seen(5, 10, 0, 1).tolist() == [5]
    assert orc.seen(5, 10, 2, 3).tolist() == [0, 1, 3, 4, 5]
    assert orc.seen(3, 10, 2, 3).tolist() == [0, 1, 2, 3]
    assert orc.seen(1, 10, 5, 1).tolist() == [0, 1]                # no sink behind oneself
    assert orc.seen(9, 10, 0, 100).tolist() == list(range(10))
    assert orc.seen(-1, 10, 4, 4).tolist() == []
    assert orc.seen(6, 10, 7, 2).tolist() == list(range(7))


def test_a_window_of_one_token_is_its_value():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((20, 4, 128)), *(rng.standard_normal((20, 2, 128)) for _ in "kv")
    got = orc.window_attention(q, k, v, [0, 7, 20], 0, 1, [0, 0, 1, 1])
    np.testing.assert_allclose(got.out, v[:, [0, 0, 1, 1]], rtol=1e-12)
    np.testing.assert_allclose(got.lse, np.einsum("thd,thd->ht", q, k[:, [0, 0, 1, 1]]) / np.sqrt(128), rtol=1e-12)


def test_a_long_window_is_causal_attention():
    rng = np.random.default_rng(2)
    q, k, v = (rng.standard_normal((30, 1, 128)) for _ in range(3))
    got = orc.window_attention(q, k, v, [0, 30], 0, 30, [0])
    z = q[:, 0] @ k[:, 0].T / np.sqrt(128) + np.triu(np.full((30, 30), -np.inf), 1)
    p = np.exp(z)
    np.testing.assert_allclose(got.out[:, 0], p @ v[:, 0] / p.sum(1, keepdims=True), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(got.lse[0], np.log(p.sum(1)), rtol=1e-10)


def _cache(rng, lens, block=64, fmt=cache_oracle.INT8):
    lens = np.asarray(lens, np.int32)
    table = np.arange(lens.size * 4, dtype=np.int32).reshape(*lens.shape, 4)
    pages = lambda: rng.integers(0, 256, size=(lens.size * 4, block, 128)).astype(np.uint8)
    return cache_oracle.CacheState(pages(), pages(), np.full(lens.size * 4, 0.25), np.full(lens.size * 4, 2.0), table, lens, fmt)


def test_windows_over_the_cache_are_those_of_its_values():
    rng = np.random.default_rng(3)
    c = _cache(rng, [[200, 70], [3, 256]])
    q = rng.standard_normal((5, 4, 128)) * 0.01
    got = orc.cache_window(c, q, [0, 3, 5], [0, 0, 1, 1], 2, 40)
    for s, h in ((0, 0), (1, 1)):
        n, rows = int(c.lens[s, h]), [0, 1, 2] if s == 0 else [3, 4]
        k, v = c.values("k", s, h, n)[:, None], c.values("v", s, h, n)[:, None]
        full = np.zeros((n, 1, 128))
        full[n - len(rows):, 0] = q[rows, 2 * h]
        want = orc.window_attention(full, k, v, [0, n], 2, 40, [0])
        np.testing.assert_allclose(got.out[rows, 2 * h], want.out[n - len(rows):, 0], rtol=1e-10)
        np.testing.assert_allclose(got.lse[2 * h, rows], want.lse[0, n - len(rows):], rtol=1e-10)
    # rows in front of a head's first token see nothing: three tokens, of which the step has two more than there are
    got = orc.cache_window(_cache(rng, [[1]]), q[:3, :1], [0, 3], [0], 0, 5)
    assert (got.out[:2] == 0).all() and np.isneginf(got.lse[0, :2]).all() and np.isfinite(got.lse[0, 2])


@pytest.mark.parametrize("alone", [False, True])
def test_a_prefix_is_what_lies_in_front(alone):
    rng = np.random.default_rng(4)
    prefix, c = _cache(rng, [[100, 30]]), _cache(rng, [[9, 9], [20, 20], [64, 64]])
    q = rng.standard_normal((4, 2, 128)) * 0.01
    got = orc.cache_shared(prefix, [0, 0] if alone else [1, 3], c, q, [0, 1, 3, 4], [0, 1])
    for row, s, back in ((0, 0, 0), (1, 1, 1), (2, 1, 0), (3, 2, 0)):
        for h in range(2):
            k, v = (c.values(x, s, h, int(c.lens[s, h]) - back) for x in "kv")
            if s > 0 and not alone:
                pk, pv = (prefix.values(x, 0, h, int(prefix.lens[0, h])) for x in "kv")
                k, v = np.concatenate([pk, k]), np.concatenate([pv, v])
            z = k @ q[row, h] / np.sqrt(128)
            p = np.exp(z - z.max())
            np.testing.assert_allclose(got.out[row, h], p @ v / p.sum(), rtol=1e-10)
            np.testing.assert_allclose(got.lse[h, row], z.max() + np.log(p.sum()), rtol=1e-10)
