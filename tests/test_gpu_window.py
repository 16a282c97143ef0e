"""GPU parity of attention with a sliding window and first tokens that stay visible, through the C ABI against the oracle."""
import numpy as np
import pytest
import torch

import paper_2603_10353_amd as S
from cache_harness import D, DEV, bf16
from oracle import window_oracle as orc
from window_harness import check

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8                               # probabilities in bf16


def stream():
    return torch.cuda.current_stream()


def inputs(rng, T, hq, hkv, pull=2.0):
    """Queries that look for some keys, the first one of all among them."""
    direction = rng.standard_normal((hkv, D))
    direction *= 4 / np.linalg.norm(direction, axis=1, keepdims=True)
    q = rng.standard_normal((T, hq, D)) + 0.5 * direction[np.arange(hq) * hkv // hq]
    k = rng.standard_normal((T, hkv, D)) + np.where(rng.random((T, hkv, 1)) < 0.03, pull, 0.0) * direction
    k[0] += 3 * direction
    return bf16(q), bf16(k), bf16(rng.standard_normal((T, hkv, D)))


def call(problem, n_sink, window, q, k, v, lse=True):
    out = torch.full_like(q, 7.0)
    l = torch.full((q.shape[1], q.shape[0]), 7.0, device=DEV) if lse else None
    S.shplb_window_attn_prefill(problem, n_sink, window, q, k, v, out, l, stream())
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), None if l is None else l.double().cpu().numpy()


def up(*pairs):
    return [p[0].to(DEV) for p in pairs]


SIZES = [  # lengths, heads, sinks, window
    ([1], 4, 4, 0, 1), ([1], 3, 1, 5, 7), ([2, 1, 3], 4, 2, 1, 1), ([63], 2, 2, 0, 63), ([64], 2, 1, 0, 64), ([65], 2, 1, 3, 64),
    ([127, 128, 129], 4, 2, 4, 100), ([300], 4, 1, 0, 1), ([300], 4, 1, 1, 1), ([300], 2, 2, 64, 64), ([300], 2, 2, 65, 127),
    ([400], 2, 1, 128, 128), ([400], 2, 1, 0, 129), ([500], 2, 2, 200, 10), ([500], 2, 1, 7, 1000), ([500], 2, 1, 1000, 3),
    ([700], 4, 2, 4, 256), ([640], 2, 2, 0, 191), ([640], 2, 2, 0, 192), ([640], 2, 2, 0, 193), ([1, 640, 64, 200, 5, 77], 7, 1, 4, 65),
    ([900], 2, 1, 2 ** 31 - 1, 2 ** 31 - 1), ([900], 2, 1, 33, 2 ** 31 - 1), ([1300], 2, 1, 100, 500),
]


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("large", [False, True], ids=["few_rows", "many_rows"])
def test_sizes(case, large):
    """As a call of few rows, and with so many sequences beside them that the call is a large one."""
    lens, hq, hkv, n_sink, window = SIZES[case]
    rng = np.random.default_rng([case, 1])
    more = []
    if large:                                  # rows of 128 queries: more than there are compute units
        more = [260 * 128 // hq // 2 + 128, 260 * 128 // hq // 2 + 5]
    cu = np.concatenate([[0], np.cumsum(lens + more)])
    (q, q64), (k, k64), (v, v64) = inputs(rng, int(cu[-1]), hq, hkv)
    out, lse = call(S.Problem(cu, hq, hkv, 128), n_sink, window, *up((q,), (k,), (v,)))
    n = int(cu[len(lens)])
    kv_of = np.arange(hq) * hkv // hq
    want = orc.window_attention(q64[:n], k64[:n], v64[:n], cu[:len(lens) + 1], n_sink, window, kv_of)
    check(want, out, lse, slice(0, n), max(lens), HALF)
    if large:                                  # the last rows of the others, too
        s = len(lens) + 1
        a, b = int(cu[s]), int(cu[s + 1])
        full = orc.Result(q64[a:b])
        rows = [0, 1, 127, 128, b - a - 1]
        for p in rows:
            at = a + orc.seen(p, b - a, n_sink, window)
            for h in range(hq):
                full.put(p, h, q64[a + p, h], k64[at, kv_of[h]], v64[at, kv_of[h]], D ** -0.5, False)
        check(full, out[a:b], lse[:, a:b], rows, b - a, HALF)


@pytest.mark.parametrize("block", [64, 128])
def test_strides_mapped_heads_scale_and_no_lse(block):
    rng = np.random.default_rng(5)
    lens, hq, hkv, kv_of = [200, 333, 1], 5, 3, [2, 0, 0, 2, 1]
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1])
    (q, q64), (k, k64), (v, v64) = inputs(rng, T, hq, 1)[0], *(bf16(rng.standard_normal((T, hkv, D))) for _ in "kv")
    qkv = torch.zeros((T, hq + 2 * hkv, D + 8), dtype=torch.bfloat16, device=DEV)
    qkv[:, :hq, :D], qkv[:, hq:hq + hkv, :D], qkv[:, hq + hkv:, :D] = q.to(DEV), k.to(DEV), v.to(DEV)
    stride = (hq + 2 * hkv) * (D + 8)
    p = S.Problem(cu, hq, hkv, block, q_stride_t=stride, q_stride_h=D + 8, kv_stride_t=stride, kv_stride_h=D + 8, softmax_scale=0.2,
                  kv_head_of=kv_of)
    out = torch.full((T, hq + 2 * hkv, D + 8), 3.0, dtype=torch.bfloat16, device=DEV)
    S.shplb_window_attn_prefill(p, 2, 90, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], out, None, stream())
    want = orc.window_attention(q64, k64, v64, cu, 2, 90, kv_of, 0.2)
    check(want, out[:, :hq, :D].double().cpu().numpy(), None, slice(0, T), 333, HALF)
    assert (out[:, hq:] == 3).all() and (out[:, :, D:] == 3).all()


@pytest.mark.parametrize("hq", [2, 64], ids=["few_rows", "many_rows"])
def test_what_is_not_finite_reaches_those_who_see_it(hq):
    rng = np.random.default_rng(9)
    T, n_sink, window = 700, 3, 130
    (q, _), (k, _), (v, _) = inputs(rng, T, hq, 2)
    v[200, 0, 5], v[201, 0, 5], v[202, 0, 77], v[350, 1, 0] = np.inf, -np.inf, np.nan, np.inf
    v[1, 1, 9] = np.nan                        # a sink: all that come after
    k[430, 0, 3] = np.nan
    k[500, 1] = np.inf
    out, lse = call(S.Problem([0, T], hq, 2, 128), n_sink, window, q.to(DEV), k.to(DEV), v.to(DEV))
    heads = [0, hq - 1]
    want = orc.window_attention(q[:, heads].double().numpy(), k.double().numpy(), v.double().numpy(), [0, T], n_sink, window, [0, 1])
    assert np.isnan(want.out[:, 0]).any(1).sum() > 200 and np.isfinite(want.out[:, 0]).all(1).sum() > 200
    assert np.isinf(want.out).any()
    check(want, out[:, heads], lse[heads], slice(0, T), T, HALF)


@pytest.mark.parametrize("T,window", [(2, 1), (5, 2), (65, 3), (130, 64), (260, 100)])
def test_what_is_not_finite_in_short_sequences(T, window):
    """... beside one without: the first token, hidden from all but a few, the last one, which nobody else sees, and one in between."""
    rng = np.random.default_rng([15, T])
    (q, q64), (k, k64), (v, _) = inputs(rng, 2 * T, 2, 1)
    v[0, 0, 3], v[T - 1, 0, 4], v[T // 2, 0, 100] = np.nan, np.inf, -np.inf
    out, lse = call(S.Problem([0, T, 2 * T], 2, 1, 128), 0, window, *up((q,), (k,), (v,)))
    want = orc.window_attention(q64, k64, v.double().numpy(), [0, T, 2 * T], 0, window, [0, 0])
    assert np.isfinite(want.out[T:]).all() and np.isnan(want.out[0, :, 3]).all() and np.isfinite(want.out[:T - 1, :, 4]).all()
    check(want, out, lse, slice(0, 2 * T), T, HALF)


def test_rows_so_far_apart_that_offsets_pass_32_bits():
    rng = np.random.default_rng(13)
    T, hq, hkv, stride = 300, 2, 1, 2 ** 24 - 8                  # a token every 32 MB
    (q, q64), (k, k64), (v, v64) = inputs(rng, T, hq, hkv)
    room = torch.empty((T - 1) * stride + 6 * D, dtype=torch.bfloat16, device=DEV)
    assert room.numel() * 2 > 2 ** 33
    at = lambda first, heads: room.as_strided((T, heads, D), (stride, D, 1), first * D)
    dq, dk, dv, out = at(0, 2), at(2, 1), at(3, 1), at(4, 2)
    dq.copy_(q), dk.copy_(k), dv.copy_(v)
    lse = torch.zeros((hq, T), device=DEV)
    p = S.Problem([0, T], hq, hkv, 128, q_stride_t=stride, q_stride_h=D, kv_stride_t=stride, kv_stride_h=D)
    S.shplb_window_attn_prefill(p, 3, 100, dq, dk, dv, out, lse, stream())
    got = out.double().cpu().numpy(), lse.double().cpu().numpy()
    check(orc.window_attention(q64, k64, v64, [0, T], 3, 100, [0, 0]), *got, slice(0, T), T, HALF)


@pytest.mark.parametrize("hq", [1, 8], ids=["few_rows", "many_rows"])
def test_as_many_sequences_as_there_may_be(hq):
    """... some of whose queries are NaN, which is nothing to the others."""
    rng = np.random.default_rng(14)
    lens = [1 + 37 * x % 130 for x in range(64)]
    cu = np.concatenate([[0], np.cumsum(lens)])
    (q, _), (k, k64), (v, v64) = inputs(rng, int(cu[-1]), hq, 1)
    q[5::41, 0, 9] = np.nan
    out, lse = call(S.Problem(cu, hq, 1, 64), 2, 50, *up((q,), (k,), (v,)))
    want = orc.window_attention(q.double().numpy(), k64, v64, cu, 2, 50, [0] * hq)
    assert np.isnan(want.out[5, 0]).all() and np.isfinite(want.out[6]).all()
    check(want, out, lse, slice(0, int(cu[-1])), max(lens), HALF)


def test_scores_of_every_size():
    """References that rise late and by far, scores far below the first tile's, queries and keys of large numbers."""
    rng = np.random.default_rng(10)
    T = 600
    for case in range(5):
        q, k, v = (rng.standard_normal((T, 2, D)) for _ in range(3))
        if case == 0:
            k *= np.linspace(0.1, 20, T)[:, None, None]          # rises again and again
        elif case == 1:
            k = np.repeat(rng.standard_normal((1, 2, D)), T, 0)   # the first tokens far below 0 for all
            q = -q.__abs__() * np.sign(k) * np.where(np.arange(T) < 300, 12, -12)[:, None, None]
        elif case == 2:
            q *= 200
        elif case == 3:
            q[:], k[:] = 0, 0
        else:
            k[::7] *= 30
        (q, q64), (k, k64), (v, v64) = bf16(q), bf16(k), bf16(v)
        for n_sink, window in ((0, 70), (4, 333)):
            out, lse = call(S.Problem([0, T], 2, 2, 128), n_sink, window, q.to(DEV), k.to(DEV), v.to(DEV))
            check(orc.window_attention(q64, k64, v64, [0, T], n_sink, window, [0, 1]), out, lse, slice(0, T), T, HALF)


def test_repeats_streams_and_graphs():
    rng = np.random.default_rng(11)
    T, hq, hkv = 3000, 16, 4
    q, k, v = up(*inputs(rng, T, hq, hkv))
    p = S.Problem([0, 1000, T], hq, hkv, 128)
    want, lse = call(p, 4, 700, q, k, v)
    out, l = torch.zeros_like(q), torch.zeros((hq, T), device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    S.shplb_window_attn_prefill(p, 4, 700, q, k, v, out, l, side)
    torch.cuda.synchronize()
    assert (out.double().cpu().numpy() == want).all() and (l.double().cpu().numpy() == lse).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.shplb_window_attn_prefill(p, 4, 700, q, k, v, out, l, stream())
    for x in range(3):
        q.copy_(torch.randn_like(q))
        graph.replay()
        a, b = out.clone(), l.clone()
        want, lse = call(p, 4, 700, q, k, v)
        assert (a.double().cpu().numpy() == want).all() and (b.double().cpu().numpy() == lse).all()


def test_a_window_no_sequence_is_longer_than_is_causal_attention():
    """Beside the selection of all blocks: the two agree within bf16's roundings of either."""
    rng = np.random.default_rng(12)
    T, hq, hkv = 1000, 4, 2
    q, k, v = up(*inputs(rng, T, hq, hkv))
    p = S.Problem([0, T], hq, hkv, 128)
    budgets = np.full(hq, 8, np.int32)
    ptr = S.shplb_sel_row_ptr(p, budgets)
    idx = torch.from_numpy(np.concatenate([np.arange(i + 1) for _ in range(hq) for i in range(8)]).astype(np.int32)).to(DEV)
    ws = torch.empty(S.shplb_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    dense, lse = torch.zeros_like(q), torch.zeros((hq, T), device=DEV)
    S.shplb_sparse_attn_prefill(p, q, k, v, torch.from_numpy(ptr).to(DEV), idx, dense, lse, None, ws, stream())
    out, l = call(p, 0, T, q, k, v)
    assert np.abs(out - dense.double().cpu().numpy()).max() <= 2e-2
    assert np.abs(l - lse.double().cpu().numpy()).max() <= 4e-3


@pytest.mark.parametrize("hq", [2, 64], ids=["few_rows", "many_rows"])
@pytest.mark.parametrize("order", ["any", "rising", "below_zero"])
@pytest.mark.parametrize("size", [10, 13, 15, 16, 20, 40, 55])
def test_scores_that_a_rounding_moves_by_more_than_one(size, order, hq):
    """Keys are whole multiples of one vector of 2^size and -2^size, queries likewise: scores are sums without rounding, multiples of 128 * 2^(2 size) *
    scale > 2^20, so that only the keys of the largest multiple that a query sees count, all alike: their probabilities are 1 / how many, what is left
    are the roundings of a probability and of the output (2^-8 each), and of the largest score, its product with the scale and the logarithm (2^-22
    of it in all)."""
    rng = np.random.default_rng([24, size])
    T, n_sink, window = 700, 3, 130
    sign = rng.choice([-1.0, 1.0], D)
    times = rng.integers(1, 100, (T, 2))
    if order == "rising":
        times = np.sort(times, 0)
    if order == "below_zero":
        times = -times
    k = times[:, :, None] * sign * 2.0 ** size
    q = rng.integers(1, 4, (T, 2, 1)) * sign * 2.0 ** size
    (q, q64), (k, k64), (v, v64) = bf16(q), bf16(k), bf16(rng.standard_normal((T, 2, D)))
    out, lse = call(S.Problem([0, T], hq, 2, 128), n_sink, window, q.repeat_interleave(hq // 2, 1).to(DEV), k.to(DEV), v.to(DEV))
    want = orc.window_attention(q64, k64, v64, [0, T], n_sink, window, [0, 1])
    heads = [0, hq - 1]
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    assert (np.abs(out[:, heads] - want.out) <= 2.0 ** -8 * np.abs(want.out) + 2.0 ** -8 * (1 + 2.0 ** -8) * want.size + 1e-30).all()
    assert (np.abs(lse[heads] - want.lse) <= 2.0 ** -22 * np.abs(want.lse)).all()
