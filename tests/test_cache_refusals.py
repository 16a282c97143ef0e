"""What the cache's entry points refuse, on the host, before any device work.  The device pointers here are never followed."""
import ctypes as C

import os

import numpy as np
import pytest

import paper_2603_10353_amd as S

FAKE = 1 << 20                     # a well-aligned address


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(S.lib_path()):
        from paper_2603_10353_amd.build import build
        build(verbose=False)


def cache(**kw):
    args = dict(k_pages=FAKE, v_pages=FAKE, k_scale=FAKE, v_scale=FAKE, page_table=FAKE, lens=FAKE, n_seq=2, n_kv_heads=4,
                block=128, max_pages=10, n_pages=100, format=S.SHPLB_CACHE_E4M3)
    args.update(kw)
    return S.Cache(**args)


def step(**kw):
    args = dict(n_seq=2, n_q_heads=8, n_kv_heads=4)
    args.update(kw)
    return S.Step(**args)


def status(call, *args):
    with pytest.raises(S.ShplbError) as e:
        call(*args)
    return e.value.status


def test_struct_layout():
    from paper_2603_10353_amd.binding import _CCache, _CStep
    assert C.sizeof(_CCache) == 80 and _CCache.k_pages.offset == 32
    assert C.sizeof(_CStep) == 72 and _CStep.n_q_heads.offset == 16 and _CStep.softmax_scale.offset == 56


@pytest.mark.parametrize("bad,code", [
    (dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1),
    (dict(page_table=None), -1), (dict(lens=None), -1), (dict(n_seq=0), -2), (dict(n_kv_heads=0), -2), (dict(max_pages=0), -2),
    (dict(n_pages=0), -2), (dict(n_pages=-1), -2), (dict(head_dim=64), -5), (dict(block=32), -5), (dict(block=256), -5),
    (dict(format=2), -5), (dict(format=-1), -5), (dict(max_pages=4097), -5), (dict(n_seq=16384), -5),
    (dict(k_pages=FAKE + 8), -2), (dict(v_pages=FAKE + 1), -2), (dict(k_scale=FAKE + 2), -2), (dict(lens=FAKE + 1), -2),
    (dict(page_table=FAKE + 2), -2),
])
def test_caches(bad, code):
    c, s = cache(**bad), step(n_seq=bad.get("n_seq", 2))
    assert status(S.shplb_cache_append, c, s, FAKE, FAKE) == code
    assert status(S.shplb_cache_load, c, s, FAKE, FAKE) == code
    assert status(S.shplb_cache_attn, c, s, FAKE, FAKE, None, None, None, FAKE) == code
    assert status(S.shplb_cache_attn_workspace_bytes, c, s) == code
    assert status(S.shplb_cache_evict_workspace_bytes, c) == code
    good = cache(page_table=2 * FAKE, lens=2 * FAKE)
    assert status(S.shplb_cache_evict, c, FAKE, FAKE, 0, 0, good, 2 * FAKE, FAKE, FAKE) == code
    assert status(S.shplb_cache_evict, good, FAKE, FAKE, 0, 0, c, 2 * FAKE, FAKE, FAKE) == code


@pytest.mark.parametrize("bad,code", [
    (dict(n_tokens=-1), -2), (dict(max_tokens=-1, n_tokens=0), -2), (dict(n_tokens=3), -2), (dict(n_tokens=3, cu_tokens=FAKE + 1), -2),
])
def test_steps(bad, code):
    s = step(**bad)
    assert status(S.shplb_cache_append, cache(), s, FAKE, FAKE) == code
    assert status(S.shplb_cache_load, cache(), s, FAKE, FAKE) == code
    assert status(S.shplb_cache_attn, cache(), s, FAKE, FAKE, None, None, None, FAKE) == code
    assert status(S.shplb_cache_attn_workspace_bytes, cache(), s) == code


@pytest.mark.parametrize("strides,code", [
    (dict(kv_stride_h=120), -2), (dict(kv_stride_h=132), -2), (dict(kv_stride_t=4 * 128 - 8), -2), (dict(kv_stride_t=4 * 128 + 4), -2),
    (dict(kv_stride_t=1 << 24), -5),
])
def test_key_strides(strides, code):
    assert status(S.shplb_cache_append, cache(), step(**strides), FAKE, FAKE) == code
    assert status(S.shplb_cache_load, cache(), step(**strides), FAKE, FAKE) == code
    assert S.shplb_cache_attn_workspace_bytes(cache(), step(**strides)) > 0          # attention has no use for them


@pytest.mark.parametrize("bad,code", [
    (dict(q_stride_h=120), -2), (dict(q_stride_t=8 * 128 - 8), -2), (dict(q_stride_t=8 * 128 + 1), -2), (dict(q_stride_t=1 << 24), -5),
    (dict(softmax_scale=-1.0), -2), (dict(softmax_scale=float("nan")), -2), (dict(softmax_scale=float("inf")), -2),
    (dict(n_q_heads=6), -2), (dict(n_q_heads=0), -2), (dict(n_q_heads=5, kv_head_of=[0, 1, 2, 4, 0]), -2),
    (dict(n_q_heads=5, kv_head_of=[0, 1, -1, 3, 0]), -2), (dict(n_q_heads=300, kv_head_of=[0] * 300), -5),
    (dict(max_tokens=1 << 24, n_tokens=5, cu_tokens=FAKE), -5),
])
def test_queries(bad, code):
    s = step(**bad)
    assert status(S.shplb_cache_attn, cache(), s, FAKE, FAKE, None, None, None, FAKE) == code
    assert status(S.shplb_cache_attn_workspace_bytes, cache(), s) == code


def test_pointers_of_the_calls():
    c, s = cache(), step()
    assert status(S.shplb_cache_append, c, s, None, FAKE) == -1
    assert status(S.shplb_cache_append, c, s, FAKE, FAKE + 8) == -2
    assert status(S.shplb_cache_load, c, s, FAKE, None) == -1
    assert status(S.shplb_cache_load, c, s, FAKE + 2, FAKE) == -2
    for args, code in [((None, FAKE, None, None, None, FAKE), -1), ((FAKE, None, None, None, None, FAKE), -1),
                       ((FAKE, FAKE, None, None, None, None), -1), ((FAKE, FAKE, None, FAKE, None, FAKE), -1),
                       ((FAKE + 8, FAKE, None, None, None, FAKE), -2), ((FAKE, FAKE + 8, None, None, None, FAKE), -2),
                       ((FAKE, FAKE, FAKE + 2, None, None, FAKE), -2), ((FAKE, FAKE, None, FAKE + 1, FAKE, FAKE), -2),
                       ((FAKE, FAKE, None, None, FAKE + 1, FAKE), -2), ((FAKE, FAKE, None, None, None, FAKE + 128), -2)]:
        assert status(S.shplb_cache_attn, c, s, *args) == code, args
    to = cache(page_table=2 * FAKE, lens=2 * FAKE)
    good = [FAKE, FAKE, 0, 0, to, 2 * FAKE, FAKE, FAKE]
    for at, value, code in [(0, None, -1), (1, None, -1), (5, None, -1), (6, None, -1), (7, None, -1), (2, -1, -3), (3, -1, -3),
                            (5, FAKE, -2), (0, FAKE + 1, -2), (1, FAKE + 2, -2), (5, FAKE + 1, -2), (6, FAKE + 3, -2), (7, FAKE + 64, -2),
                            (4, cache(), -2), (4, cache(page_table=2 * FAKE), -2), (4, cache(lens=2 * FAKE), -2),
                            (4, cache(page_table=2 * FAKE, lens=2 * FAKE, n_seq=3), -2),
                            (4, cache(page_table=2 * FAKE, lens=2 * FAKE, n_kv_heads=2), -2),
                            (4, cache(page_table=2 * FAKE, lens=2 * FAKE, format=S.SHPLB_CACHE_INT8), -2)]:
        args = list(good)
        args[at] = value
        assert status(S.shplb_cache_evict, c, *args) == code, (at, value)


def test_output_in_place():
    # queries are read again after the first outputs are written
    assert status(S.shplb_cache_attn, cache(), step(), FAKE, FAKE, None, None, None, FAKE) == -2


def test_strides_whose_product_is_past_64_bits():
    s = step(n_tokens=2)
    s.c.kv_stride_h = s.c.q_stride_h = 1 << 62
    assert status(S.shplb_cache_append, cache(), s, FAKE, FAKE) == -2
    assert status(S.shplb_cache_load, cache(), s, FAKE, FAKE) == -2
    assert status(S.shplb_cache_attn_workspace_bytes, cache(), s) == -2


@pytest.mark.parametrize("n_seq,max_pages,max_tokens,fits", [
    (2048, 4096, 1, True), (8192, 4096, 32, True), (8192, 4096, 224, True), (8192, 4096, 256, False),       # units of 64 keys: below 2^30
    (4000, 1, 34000, False), (3900, 1, 34000, True),                                                     # tiles of 32 rows: below 2^24
    (4000, 58, 32000, True), (4000, 60, 32000, False),                                                   # ... and eight units more for each
])
def test_most_that_attention_takes(n_seq, max_pages, max_tokens, fits):
    c = cache(n_seq=n_seq, n_kv_heads=4, max_pages=max_pages, block=64)
    s = step(n_seq=n_seq, n_q_heads=4, n_tokens=5, max_tokens=max_tokens, cu_tokens=FAKE)
    if fits:
        assert S.shplb_cache_attn_workspace_bytes(c, s) > 0
    else:
        assert status(S.shplb_cache_attn_workspace_bytes, c, s) == -5
        assert status(S.shplb_cache_attn, c, s, FAKE, 2 * FAKE, None, None, None, FAKE) == -5


def test_most_pages_of_a_call():
    # 2^23 pages that a call may touch
    c = cache(n_seq=2048, n_kv_heads=4, max_pages=1024, block=64)
    s = step(n_seq=2048, n_tokens=5, max_tokens=1024 * 64, cu_tokens=FAKE)
    assert status(S.shplb_cache_append, c, s, FAKE, FAKE) == -5
    assert status(S.shplb_cache_load, c, s, FAKE, FAKE) == -5
    small = cache(n_seq=2048, n_kv_heads=4, max_pages=4, page_table=2 * FAKE, lens=2 * FAKE)
    assert status(S.shplb_cache_evict, small, FAKE, FAKE, 0, 0, c, 2 * FAKE, FAKE, FAKE) == -5


def test_calls_without_work_need_no_pointers():
    # a step without tokens is done before it begins
    for s in (step(n_tokens=0, max_tokens=0), step(n_tokens=0, max_tokens=3, cu_tokens=FAKE)):
        S.shplb_cache_append(cache(), s, None, None)
        S.shplb_cache_load(cache(), s, None, None)
        S.shplb_cache_attn(cache(), s, None, None, None, None, None, None)


def test_workspace_sizes():
    a = S.shplb_cache_attn_workspace_bytes(cache(), step())
    b = S.shplb_cache_attn_workspace_bytes(cache(), step(max_tokens=8))
    c = S.shplb_cache_attn_workspace_bytes(cache(), step(max_tokens=64))
    assert 0 < a <= b <= c and a % 256 == b % 256 == 0
    assert S.shplb_cache_evict_workspace_bytes(cache()) > 0
    with pytest.raises(ValueError):
        step(n_q_heads=5, kv_head_of=[0, 1])
    assert np.asarray(step(n_q_heads=5, kv_head_of=[0, 1, 2, 3, 0]).kv_head_of).size == 5


# arrays of an eviction, each at an address of its own
EVICT_ARRAYS = ["lens", "table", "to_lens", "to_table", "weight", "keep", "weight_out", "kept_out", "workspace"]


@pytest.mark.parametrize("written,other", [(x, y) for x in ("to_lens", "weight_out", "kept_out", "workspace") for y in EVICT_ARRAYS if x != y])
def test_arrays_that_eviction_writes_are_no_others(written, other):
    # budgets, lengths, weights and positions are read while others' lengths, weights and positions are written
    at = {x: (i + 2) * FAKE for i, x in enumerate(EVICT_ARRAYS)}
    at[written] = at[other]
    to = cache(page_table=at["to_table"], lens=at["to_lens"])
    assert status(S.shplb_cache_evict, cache(page_table=at["table"], lens=at["lens"]), at["weight"], at["keep"], 1, 1, to,
                  at["weight_out"], at["kept_out"], at["workspace"]) == -2
