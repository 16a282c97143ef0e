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
