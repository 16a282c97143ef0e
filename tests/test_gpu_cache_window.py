"""GPU parity of attention with a sliding window over the 8-bit cache, through the C ABI against the oracle."""
import numpy as np
import pytest
import torch

import paper_2603_10353_amd as S
from cache_harness import D, DEV, Device, bf16, filled, step_of, strided
from oracle import cache_oracle, window_oracle as orc
from window_harness import check, check_far, far_apart, in_a_large_pool

pytestmark = pytest.mark.gpu
FORMATS = pytest.mark.parametrize("fmt", [cache_oracle.E4M3, cache_oracle.INT8], ids=["e4m3", "int8"])
HALF, LIFT = 2.0 ** -11, 2.0 ** -32            # probabilities in fp16, held at 2^7 times their size


def stream():
    return torch.cuda.current_stream()


def workspace(dev, step, n_sink, window):
    return torch.empty(S.shplb_cache_attn_window_workspace_bytes(dev.cache, step, n_sink, window), dtype=torch.uint8, device=DEV).fill_(0xff)


def call(dev, step, n_sink, window, q, ws=None, on=None):
    out, lse = torch.full_like(q, 7.0), torch.full((q.shape[1], q.shape[0]), 7.0, device=DEV)
    S.shplb_cache_attn_window(dev.cache, step, n_sink, window, q, out, lse, workspace(dev, step, n_sink, window) if ws is None else ws, on or stream())
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def forget(rng, c, new, n_sink, window):
    """Table entries of pages that no row needs become anything, what lies in front of all windows in the others NaN."""
    for s in range(c.table.shape[0]):
        for h in range(c.table.shape[1]):
            n = int(c.lens[s, h])
            low = max(0, n - int(new[s]) + 1 - window)
            if new[s] == 0:
                low = n
            hidden = np.arange(min(n_sink, n), low)
            for i in range(c.table.shape[2]):
                in_page = np.arange(i * c.block, (i + 1) * c.block)
                held = in_page[in_page < n]
                if held.size and np.isin(held, hidden).all():
                    c.table[s, h, i] = rng.choice([-1, -2 ** 31, c.n_pages, 2 ** 31 - 1, int(c.table[s, h, i])])
                elif held.size:
                    for pages in (c.k_pages, c.v_pages):
                        pages[c.table[s, h, i], np.isin(in_page, hidden)] = 0x7f if c.fmt == cache_oracle.E4M3 else 0x80


CASES = {  # lengths, new tokens, query heads, KV heads, sinks, window
    "one_token": ([[1], [2], [64], [65]], [1, 1, 1, 1], 4, 1, 0, 1),
    "small": ([[300, 40], [7, 128], [129, 640]], [1, 1, 1], 8, 2, 4, 100),
    "edges": ([[n] for n in (1, 63, 64, 65, 127, 128, 129, 191, 192, 193, 256, 500)], [1] * 12, 4, 1, 64, 64),
    "edges_of_windows": ([[n] for n in (1, 63, 64, 65, 127, 128, 129, 191, 192, 193, 256, 500)], [1] * 12, 4, 1, 3, 65),
    "no_sink": ([[700, 333]], [1], 2, 2, 0, 128),
    "all_sinks": ([[700, 333]], [1], 2, 2, 2 ** 31 - 1, 5),
    "more_sinks_than_window": ([[700, 333], [90, 1]], [1, 1], 2, 2, 200, 3),
    "long_window": ([[700, 333]], [1], 2, 2, 7, 2 ** 31 - 1),
    "tokens": ([[300, 40], [7, 128], [129, 640], [50, 60]], [4, 2, 1, 0], 8, 2, 4, 60),
    "more_tokens_than_held": ([[3, 200], [0, 1]], [4, 4], 4, 2, 2, 70),
    "rows_32": ([[300, 400]], [16], 4, 2, 5, 90),
    "rows_of_many_tiles": ([[700], [90]], [100, 77], 3, 1, 70, 130),
    "by_shares": ([[5000, 300], [2, 3500]], [1, 1], 4, 2, 130, 2600),
    "by_shares_tokens": ([[4500, 300], [2900, 3500]], [5, 2], 4, 2, 4, 2500),
    "by_shares_rows": ([[4700, 6000]], [20], 4, 2, 64, 4100),
    "wide": ([[700, 65], [300, 500]], [40, 64], 8, 2, 4, 100),
    "wide_sinks": ([[700], [90], [64]], [100, 77, 3], 3, 1, 200, 130),
    "wide_whole_prompts": ([[200], [150], [64]], [200, 150, 64], 2, 1, 0, 31),
    "wide_long": ([[6000, 9000]], [70], 4, 2, 130, 4100),
    "wide_more_than_held": ([[30, 200], [0, 1], [100, 100]], [64, 40, 0], 4, 2, 2, 70),
    "wide_everything": ([[1500]], [60], 4, 1, 0, 2 ** 31 - 1),
    "wide_uneven_groups": ([[260, 300, 10]], [25], 21, 3, 1, 70),
    "groups_of_seven": ([[260, 300, 10]], [3], 21, 3, 1, 70),
}


@FORMATS
@pytest.mark.parametrize("block", [128, 64])
@pytest.mark.parametrize("name", CASES)
def test_sizes(name, block, fmt):
    lens, new, hq, hkv, n_sink, window = CASES[name]
    assert len(lens[0]) == hkv
    rng = np.random.default_rng([fmt, block, len(name)])
    c = filled(rng, lens, block, fmt, max_pages=60 if name == "small" else None)
    new = np.array(new)
    ragged = len(set(new.tolist())) > 1
    forget(rng, c, new, n_sink, window)
    dev = Device(c)
    T = int(new.sum())
    q, q64 = bf16(rng.standard_normal((T, hq, D)))
    step, cu = step_of(dev, new, hq, ragged)
    out, lse = call(dev, step, n_sink, window, q.to(DEV))
    kv_of = np.arange(hq) * hkv // hq
    check(orc.cache_window(c, q64, cu, kv_of, n_sink, window), out, lse, slice(0, T), int(np.max(lens)), HALF, LIFT)


@FORMATS
def test_a_batch_of_many_heads(fmt):
    """More heads than a wave adds up by itself, windows longer and shorter than the sequences."""
    rng = np.random.default_rng(3)
    n, hkv = 150, 4
    lens = rng.integers(1, 200, size=(n, hkv))
    lens[7], lens[100, 2] = 2900, 3300
    c = filled(rng, lens, 128, fmt)
    new = np.ones(n, np.int64)
    forget(rng, c, new, 4, 2300)
    dev = Device(c)
    q, q64 = bf16(rng.standard_normal((n, hkv, D)))
    step, cu = step_of(dev, new, hkv, False)
    out, lse = call(dev, step, 4, 2300, q.to(DEV))
    check(orc.cache_window(c, q64, cu, np.arange(hkv), 4, 2300), out, lse, slice(0, n), 3300, HALF, LIFT)


@FORMATS
def test_strides_mapped_heads_scale_rows_behind(fmt):
    rng = np.random.default_rng(4)
    kv_of = [2, 0, 0, 2, 0]                    # one KV head without query heads
    lens, new = [[100, 50, 300], [80, 1, 129]], np.array([2, 3])
    c = filled(rng, lens, 64, fmt)
    dev = Device(c)
    q, q64 = bf16(rng.standard_normal((7, 5, D)))
    qd, wide = strided(q, 4)
    step, cu = step_of(dev, new, 5, True, behind=2, q_stride_t=wide.shape[1] * D, softmax_scale=0.2, kv_head_of=kv_of)
    out = torch.full_like(wide, 5.0)
    S.shplb_cache_attn_window(dev.cache, step, 3, 50, qd, out[:, 2:7], None, workspace(dev, step, 3, 50), stream())
    want = orc.cache_window(c, q64, cu, kv_of, 3, 50, 0.2)
    check(want, out[:, 2:7].double().cpu().numpy(), None, slice(0, 5), 300, HALF, LIFT)
    assert (out[5:] == 5).all() and (out[:, :2] == 5).all() and (out[:, 7:] == 5).all()


@FORMATS
@pytest.mark.parametrize("wide", [False, True])
def test_damage_reaches_those_who_see_it(fmt, wide):
    """Lengths that cannot be, pages that are not there, pages with a scale of NaN: eight tokens, of which the first see the page
    that is damaged, and the last do not."""
    rng = np.random.default_rng(5)
    group = 12 if wide else 1
    lens = [[300], [-1], [1000], [300], [300], [300]]
    c = filled(rng, np.clip(lens, 0, 384), 64, fmt, max_pages=6)
    c.lens[:] = lens
    c.table[3, 0, 2] = -1                      # positions 128 .. 191; windows of 108: the last tokens begin behind
    c.k_scale[c.table[4, 0, 2]] = np.nan
    c.v_scale[c.table[5, 0, 2]] = np.nan
    for s in (3, 4, 5):
        c.table[s, 0, 1] = 10 ** 6
    dev = Device(c)
    q, q64 = bf16(rng.standard_normal((48, group, D)))
    step, cu = step_of(dev, [8] * 6, group, False)
    want = orc.cache_window(c, q64, cu, [0] * group, 4, 105)
    assert np.isnan(want.out[24:28]).all() and np.isfinite(want.out[28:32]).all() and np.isnan(want.out[8:24]).all()
    check(want, *call(dev, step, 4, 105, q.to(DEV)), slice(0, 48), 384, HALF, LIFT)


def test_large_scales_and_queries():
    """Pages whose scales leave fp16, queries in the hundreds of thousands, references that rise late."""
    rng = np.random.default_rng(6)
    for size, qsize in ((2.0 ** 40, 2.0 ** -40), (2.0 ** -60, 2.0 ** 60), (1.0, 300.0), (2.0 ** -100, 1.0)):
        c = filled(rng, [[500, 3000]], 128, cache_oracle.E4M3, size=size)
        dev = Device(c)
        for n in (3, 60):
            q, q64 = bf16(rng.standard_normal((n, 2, D)) * qsize)
            step, cu = step_of(dev, [n], 2, False)
            for window in (100, 2500):
                want = orc.cache_window(c, q64, cu, [0, 1], 2, window)
                check(want, *call(dev, step, 2, window, q.to(DEV)), slice(0, n), 3000, HALF, LIFT)


@pytest.mark.parametrize("new", [1, 12, 50])
def test_a_pool_past_32_bits_and_queries_of_nan(new):
    rng = np.random.default_rng(21)
    lens = [[900, 333], [70, 60], [500, 129]]
    c = filled(rng, lens, 128, cache_oracle.E4M3)
    dev = in_a_large_pool(c)
    q, _ = bf16(rng.standard_normal((3 * new, 4, D)))
    q[new, 1, 77] = np.nan
    step, cu = step_of(dev, [new] * 3, 4, False)
    want = orc.cache_window(c, q.double().numpy(), cu, [0, 0, 1, 1], 5, 200)
    assert np.isnan(want.out[new, 1]).all() and np.isfinite(want.out[new, 0]).all()
    check(want, *call(dev, step, 5, 200, q.to(DEV)), slice(0, 3 * new), 900, HALF, LIFT)


@pytest.mark.parametrize("window", [50, 2500])
def test_graph_of_a_step_streams_and_workspaces(window):
    """A captured step stays right while lengths, table and windows' pages change; two calls at once have workspaces of their own."""
    rng = np.random.default_rng(7)
    c = filled(rng, [[3000, 200], [40, 2700]], 128, cache_oracle.INT8, spare=2)
    dev = Device(c)
    q = bf16(rng.standard_normal((2, 4, D)))[0].to(DEV)
    step, cu = step_of(dev, [1, 1], 4, False)
    ws = [workspace(dev, step, 4, window) for _ in range(2)]
    out, lse = torch.zeros_like(q), torch.zeros((4, 2), device=DEV)
    call(dev, step, 4, window, q, ws[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.shplb_cache_attn_window(dev.cache, step, 4, window, q, out, lse, ws[0], stream())
    side = torch.cuda.Stream()
    for x in range(4):
        other, other_lse = torch.zeros_like(q), torch.zeros((4, 2), device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        S.shplb_cache_attn_window(dev.cache, step, 4, window, q, other, other_lse, ws[1], side)
        torch.cuda.synchronize()
        want, want_lse = call(dev, step, 4, window, q, ws[1])
        assert (out.double().cpu().numpy() == want).all() and (other.double().cpu().numpy() == want).all()
        assert (lse.double().cpu().numpy() == want_lse).all() and (other_lse.double().cpu().numpy() == want_lse).all()
        dev.lens += 31
        q.copy_(torch.randn_like(q))


def test_a_prompt_and_the_tokens_behind_it():
    """The operators as they are used: a prompt with a window, its keys and values into the cache, tokens one by one over it, in pages
    that are used in turn."""
    rng = np.random.default_rng(8)
    T, hq, hkv, n_sink, window, block = 500, 4, 2, 4, 150, 64
    steps, pages = 90, 10
    total = T + steps
    (q, q64), (k, _), (v, _) = (bf16(rng.standard_normal((total, h, D))) for h in (hq, hkv, hkv))
    q, k, v = (x.to(DEV) for x in (q, k, v))
    out, lse = torch.zeros_like(q), torch.zeros((hq, T), device=DEV)
    S.shplb_window_attn_prefill(S.Problem([0, T], hq, hkv, 128), n_sink, window, q[:T], k[:T], v[:T], out[:T], lse, stream())
    want = orc.window_attention(q64[:T], *(x[:T].double().cpu().numpy() for x in (k, v)), [0, T], n_sink, window, np.arange(hq) // 2)
    check(want, out[:T].double().cpu().numpy(), lse.double().cpu().numpy(), slice(0, T), T, 2.0 ** -8)
    # a cache with a page for the first tokens and five more a head
    nb = -(-total // block)
    table = np.zeros((1, hkv, nb), np.int32)
    for h in range(hkv):
        for i in range(nb):
            table[0, h, i] = h * 6 + (0 if i == 0 else 1 + (i - 1) % 5)
    z = lambda: np.zeros((12, block, D), np.uint8)
    c = cache_oracle.CacheState(z(), z(), np.ones(12), np.ones(12), table, np.zeros((1, hkv), np.int32), cache_oracle.E4M3)
    dev = Device(c)
    def append(first, end):
        dev.lens.fill_(end)
        c.lens[:] = end
        S.shplb_cache_append(dev.cache, S.Step(1, hq, hkv, max_tokens=end - first), k[first:end], v[first:end], stream())
        orc_k, orc_v = (x[first:end].double().cpu().numpy() for x in (k, v))
        cache_oracle.append(c, orc_k, orc_v, [0, end - first])
    append(0, 64)
    for at in range(64, T, block):             # pages in turn: one at a time
        append(at, min(at + block, T))
    step = S.Step(1, hq, hkv)
    ws = workspace(dev, step, n_sink, window)
    for t in range(T, total):
        append(t, t + 1)
        S.shplb_cache_attn_window(dev.cache, step, n_sink, window, q[t:t + 1], out[t:t + 1], None, ws, stream())
        want = orc.cache_window(c, q64[t:t + 1], [0, 1], np.arange(hq) // 2, n_sink, window)
        check(want, out[t:t + 1].double().cpu().numpy(), None, slice(0, 1), total, HALF, LIFT)
    dev.check_same(c)


@FORMATS
@pytest.mark.parametrize("group", [1, 12], ids=["rows_8", "rows_96"])
@pytest.mark.parametrize("n_sink,window,pages", [(0, 105, 6), (0, 2 ** 31 - 1, 6), (0, 3000, 70), (5, 3000, 70)], ids=["short", "all", "by_shares", "by_shares_with_sinks"])
def test_lengths_that_cannot_be(fmt, group, n_sink, window, pages):
    """... without first tokens, too, whose unit is else the one that is looked up; heads beside them stay as they are."""
    rng = np.random.default_rng(23)
    lens = np.array([[300], [10 ** 9], [64 * pages + 1], [64 * pages], [2 ** 31 - 1], [-1], [-2 ** 30 - 3], [-2 ** 31], [300]])
    c = filled(rng, np.where((lens >= 0) & (lens <= 64 * pages), lens, 0), 64, fmt, max_pages=pages)
    c.lens[:] = lens
    dev = Device(c)
    n = 8 * len(lens)
    q, q64 = bf16(rng.standard_normal((n, group, D)))
    step, cu = step_of(dev, [8] * len(lens), group, False)
    want = orc.cache_window(c, q64, cu, [0] * group, n_sink, window)
    whole = [s for s in range(len(lens)) if np.isfinite(want.out[8 * s:8 * s + 8]).all()]
    assert whole == [0, 3, 8] and np.isnan(want.out[8:24]).all() and np.isnan(want.out[32:64]).all()
    check(want, *call(dev, step, n_sink, window, q.to(DEV)), slice(0, n), 64 * pages, HALF, LIFT)


@pytest.mark.parametrize("fmt,block", [(cache_oracle.E4M3, 128), (cache_oracle.INT8, 64)], ids=["e4m3", "int8"])
@pytest.mark.parametrize("n,new,window", [(32, 4, 2400), (64, 8, 4400), (65, 8, 4474)], ids=["128_tiles", "512_tiles", "520_tiles_of_the_longest"])
def test_tiles_of_longer_windows_a_workgroup_each(n, new, window, fmt, block):
    """Windows of more than 2048 tokens and so many tiles of 32 rows that each is a workgroup's: up to 18 units a wave.  A few sequences are long."""
    rng = np.random.default_rng([26, n])
    lens = rng.integers(1, 90, (n, 1))
    lens[[0, n // 2, n - 1], 0] = [5000, window + 1, 4700]
    c = filled(rng, lens, block, fmt)
    forget(rng, c, np.full(n, new), 3, window)
    dev = Device(c)
    q, q64 = bf16(rng.standard_normal((n * new, 32, D)))
    step, cu = step_of(dev, [new] * n, 32, False)
    out, lse = call(dev, step, 3, window, q.to(DEV))
    check(orc.cache_window(c, q64, cu, [0] * 32, 3, window), out, lse, slice(0, n * new), 5000, HALF, LIFT)


@FORMATS
@pytest.mark.parametrize("order", ["any", "rising", "below_zero"])
@pytest.mark.parametrize("size", [(10, 10), (15, 16), (16, 20), (40, 40), (100, -30), (-60, 115)])
def test_scores_that_a_rounding_moves_by_more_than_one(size, order, fmt):
    rng = np.random.default_rng([27, *(abs(x) for x in size)])
    lens = [[700, 3100], [90, 64]]
    c = filled(rng, lens, 64, fmt)
    n = np.max(lens, 1)
    cu = [0, n[0], n.sum()]
    cache_oracle.append(c, bf16(far_apart(rng, (int(n.sum()), 2), size[0], order))[1], bf16(rng.standard_normal((int(n.sum()), 2, D)))[1], cu)
    dev = Device(c)
    for new in (2, 12):
        q, q64 = bf16(far_apart(rng, (2 * new, 4), size[1], "any"))
        step, cu = step_of(dev, [new, new], 4, False)
        for window in (100, 3000):
            want = orc.cache_window(c, q64, cu, [0, 0, 1, 1], 2, window)
            check_far(want, *call(dev, step, 2, window, q.to(DEV)), slice(0, 2 * new), HALF)
