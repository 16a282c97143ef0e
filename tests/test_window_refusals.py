"""What attention with a window refuses, on the host, before any device work.  The device pointers here are never followed."""
import os

import pytest

import paper_2603_10353_amd as S

FAKE = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(S.lib_path()):
        from paper_2603_10353_amd.build import build
        build(verbose=False)


def status(call, *args):
    with pytest.raises(S.ShplbError) as e:
        call(*args)
    return e.value.status


def problem(**kw):
    args = dict(cu_seqlens=[0, 128], n_q_heads=4, n_kv_heads=2, block=128)
    args.update(kw)
    return S.Problem(**args)


@pytest.mark.parametrize("n_sink,window,code", [(-1, 1, -3), (0, 0, -3), (0, -5, -3), (-2 ** 31, 2 ** 31 - 1, -3)])
def test_windows(n_sink, window, code):
    assert status(S.shplb_window_attn_prefill, problem(), n_sink, window, FAKE, FAKE, FAKE, FAKE) == code


@pytest.mark.parametrize("at", range(4))
def test_pointers(at):
    args = [2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE]
    args[at] = None
    assert status(S.shplb_window_attn_prefill, problem(), 0, 1, *args) == -1
    args[at] = FAKE + 8
    assert status(S.shplb_window_attn_prefill, problem(), 0, 1, *args) == -2


def test_lse_alignment():
    assert status(S.shplb_window_attn_prefill, problem(), 0, 1, FAKE, FAKE, FAKE, 2 * FAKE, FAKE + 2) == -2


@pytest.mark.parametrize("at", range(3))
def test_output_in_place(at):
    args = [2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE]
    args[at] = args[3]
    assert status(S.shplb_window_attn_prefill, problem(), 0, 1, *args) == -2


@pytest.mark.parametrize("bad,code", [
    (dict(head_dim=64), -5), (dict(block=32), -5), (dict(n_q_heads=3), -2), (dict(cu_seqlens=[1, 128]), -2), (dict(cu_seqlens=[0, 128, 128]), -2),
    (dict(cu_seqlens=list(range(0, 66 * 128, 128))), -5), (dict(cu_seqlens=[0, 128 * 4097]), -5), (dict(q_stride_h=100), -2),
    (dict(kv_stride_h=132), -2), (dict(softmax_scale=-1.0), -2), (dict(softmax_scale=float("nan")), -2), (dict(q_stride_t=1 << 24), -5),
    (dict(n_q_heads=3, kv_head_of=[0, 2, 1]), -2),
])
def test_problems(bad, code):
    assert status(S.shplb_window_attn_prefill, problem(**bad), 0, 1, FAKE, FAKE, FAKE, 2 * FAKE) == code


def test_strides_whose_product_is_past_64_bits():
    p = problem()
    p.c.q_stride_h = 1 << 62
    assert status(S.shplb_window_attn_prefill, p, 0, 1, FAKE, FAKE, FAKE, 2 * FAKE) == -5


def test_no_problem():
    lib = S.load_library()
    assert lib.shplb_window_attn_prefill(None, 0, 1, FAKE, FAKE, FAKE, FAKE, None, None) == -1


# ---- over the cache -----------------------------------------------------------------------------------------------------


def cache(**kw):
    args = dict(k_pages=FAKE, v_pages=FAKE, k_scale=FAKE, v_scale=FAKE, page_table=FAKE, lens=FAKE, n_seq=2, n_kv_heads=4,
                block=128, max_pages=10, n_pages=100, format=S.SHPLB_CACHE_E4M3)
    args.update(kw)
    return S.Cache(**args)


def step(**kw):
    args = dict(n_seq=2, n_q_heads=8, n_kv_heads=4)
    args.update(kw)
    return S.Step(**args)


def window_calls(c, s):
    yield lambda: S.shplb_cache_attn_window(c, s, 0, 1, FAKE, 2 * FAKE, None, FAKE)
    yield lambda: S.shplb_cache_attn_window_workspace_bytes(c, s, 0, 1)


def shared_calls(p, c, s):
    yield lambda: S.shplb_cache_attn_shared(p, FAKE, c, s, FAKE, 2 * FAKE, None, FAKE)
    yield lambda: S.shplb_cache_attn_shared_workspace_bytes(p, c, s)


BAD_CACHES = [
    (dict(k_pages=None), -1), (dict(v_scale=None), -1), (dict(page_table=None), -1), (dict(lens=None), -1), (dict(n_seq=0), -2),
    (dict(max_pages=0), -2), (dict(n_pages=0), -2), (dict(head_dim=64), -5), (dict(block=32), -5), (dict(format=2), -5),
    (dict(max_pages=4097), -5), (dict(n_seq=16384), -5), (dict(k_pages=FAKE + 8), -2), (dict(lens=FAKE + 1), -2),
]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_caches(bad, code):
    c, s = cache(**bad), step(n_seq=bad.get("n_seq", 2))
    for call in window_calls(c, s):
        assert status(call) == code
    for call in shared_calls(cache(), c, s):
        assert status(call) == code
    for call in shared_calls(c, cache(), step()):
        assert status(call) == code


@pytest.mark.parametrize("bad,code", [
    (dict(n_tokens=-1), -2), (dict(max_tokens=-1, n_tokens=0), -2), (dict(n_tokens=3), -2), (dict(n_tokens=3, cu_tokens=FAKE + 1), -2),
    (dict(q_stride_h=120), -2), (dict(q_stride_t=8 * 128 - 8), -2), (dict(q_stride_t=8 * 128 + 1), -2), (dict(q_stride_t=1 << 24), -5),
    (dict(softmax_scale=-1.0), -2), (dict(softmax_scale=float("nan")), -2), (dict(n_q_heads=6), -2), (dict(n_q_heads=0), -2),
    (dict(n_q_heads=5, kv_head_of=[0, 1, 2, 4, 0]), -2), (dict(n_q_heads=300, kv_head_of=[0] * 300), -5),
    (dict(max_tokens=1 << 24, n_tokens=5, cu_tokens=FAKE), -5),
])
def test_steps(bad, code):
    for call in (*window_calls(cache(), step(**bad)), *shared_calls(cache(), cache(), step(**bad))):
        assert status(call) == code


@pytest.mark.parametrize("n_sink,window", [(-1, 1), (0, 0), (0, -7)])
def test_windows_over_the_cache(n_sink, window):
    assert status(S.shplb_cache_attn_window, cache(), step(), n_sink, window, FAKE, 2 * FAKE, None, FAKE) == -3
    assert status(S.shplb_cache_attn_window_workspace_bytes, cache(), step(), n_sink, window) == -3


@pytest.mark.parametrize("args,code", [
    ((None, FAKE, None, FAKE), -1), ((FAKE, None, None, FAKE), -1), ((FAKE, 2 * FAKE, None, None), -1), ((FAKE, FAKE, None, FAKE), -2),
    ((FAKE + 8, FAKE, None, FAKE), -2), ((FAKE, FAKE + 8, None, FAKE), -2), ((FAKE, 2 * FAKE, FAKE + 2, FAKE), -2), ((FAKE, 2 * FAKE, None, FAKE + 128), -2),
])
def test_pointers_over_the_cache(args, code):
    assert status(S.shplb_cache_attn_window, cache(), step(), 0, 1, *args) == code
    assert status(S.shplb_cache_attn_shared, cache(), FAKE, cache(), step(), *args) == code


def test_prefixes():
    assert status(S.shplb_cache_attn_shared, cache(), None, cache(), step(), FAKE, 2 * FAKE, None, FAKE) == -1
    assert status(S.shplb_cache_attn_shared, cache(), FAKE + 2, cache(), step(), FAKE, 2 * FAKE, None, FAKE) == -2
    for call in shared_calls(cache(n_kv_heads=2), cache(), step()):
        assert status(call) == -2
    lib = S.load_library()
    assert lib.shplb_cache_attn_shared_workspace_bytes(cache().ref(), cache().ref(), step().ref(), None) == -1
    for call in shared_calls(cache(format=S.SHPLB_CACHE_INT8), cache(), step()):
        assert status(call) == -2
    # other blocks and numbers of sequences than the prefixes' are fine
    other = cache(block=64, n_seq=7)
    assert S.shplb_cache_attn_shared_workspace_bytes(other, cache(), step()) > 0


def test_limits():
    # all rows of a KV head may have the same prefix: 2^24 at most, and units of 64 tokens for every tile of them below 2^30
    many = step(n_seq=2, n_tokens=2 * ((1 << 22) + 1), max_tokens=(1 << 22) + 1)
    for call in shared_calls(cache(), cache(), many):
        assert status(call) == -5
    long = cache(max_pages=4096, n_seq=1)
    for tokens, fits in ((1 << 12, True), (1 << 20, False)):
        s = step(n_tokens=2 * tokens, max_tokens=tokens)
        if fits:
            assert S.shplb_cache_attn_shared_workspace_bytes(long, cache(), s) > 0
        else:
            assert status(S.shplb_cache_attn_shared_workspace_bytes, long, cache(), s) == -5


def test_nothing_to_do():
    """Steps without tokens touch nothing."""
    s = step(n_tokens=0, max_tokens=0)
    S.shplb_cache_attn_window(cache(), s, 0, 1, None, None, None, None)
    S.shplb_cache_attn_shared(cache(), None, cache(), s, None, None, None, None)


def test_a_workspace_for_more_tokens_does_for_fewer():
    sizes = []
    for n in (1, 2, 3, 5, 8, 9, 16, 17, 33, 60, 100, 257, 600):
        s = step(n_tokens=2 * n, max_tokens=n)
        sizes.append((S.shplb_cache_attn_window_workspace_bytes(cache(), s, 4, 100),
                      *(S.shplb_cache_attn_shared_workspace_bytes(cache(max_pages=m), cache(), s) for m in (1, 100, 4096))))
    for a, b in zip(sizes, sizes[1:]):
        assert all(x <= y for x, y in zip(a, b))
