"""GPU parity of the 8-bit key/value cache through the C ABI against the oracle: codes and scales byte for byte, attention within
tolerances made of its roundings (cache_harness.check_attn)."""
import numpy as np
import pytest
import torch

import paper_2603_10353_amd as S
from cache_harness import D, DEV, Device, attn_workspace, bf16, check_attn, filled, state, step_of, strided
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu
FORMATS = pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8], ids=["e4m3", "int8"])
BLOCKS = pytest.mark.parametrize("block", [128, 64])


def stream():
    return torch.cuda.current_stream()


# ---- append and load ----------------------------------------------------------------------------------------------------

# tokens held after the call, and how many of them are new
APPENDS = {
    "one_of_one": ([1], [1]),
    "prompts": ([1, 63, 64, 65, 127, 128, 129, 300], [1, 63, 64, 65, 127, 128, 129, 300]),
    "steps": ([1, 2, 64, 65, 128, 129, 200, 256], [1] * 8),
    "pieces": ([200, 65, 128, 129, 500, 3, 64, 300], [100, 64, 1, 2, 0, 3, 63, 290]),
    "none_but_one": ([100, 0, 70], [0, 0, 6]),
}


@FORMATS
@BLOCKS
@pytest.mark.parametrize("name", APPENDS)
def test_append_and_load(name, block, fmt):
    lens, new = (np.array(x) for x in APPENDS[name])
    rng = np.random.default_rng([block, fmt, len(name)])
    hkv, packed = 3, name in ("prompts", "pieces")
    c = filled(rng, np.repeat((lens - new)[:, None], hkv, 1), block, fmt, max_pages=-(-int(lens.max()) // block) + 1)
    used = set(c.table[c.table >= 0].tolist())
    for s in range(lens.size):                           # pages for what comes
        for h in range(hkv):
            for i in range(-(-int(lens[s]) // block)):
                if c.table[s, h, i] < 0:
                    c.table[s, h, i] = max(used) + 1
                    used.add(int(c.table[s, h, i]))
    more = max(used) + 1 - c.n_pages
    if more > 0:
        pad = lambda a: np.concatenate([a, rng.integers(0, 256, size=(more, block, D)).astype(np.uint8)])
        c.k_pages, c.v_pages = pad(c.k_pages), pad(c.v_pages)
        c.k_scale, c.v_scale = np.concatenate([c.k_scale, np.ones(more)]), np.concatenate([c.v_scale, np.ones(more)])
    c.lens[:] = lens[:, None]
    dev = Device(c)
    ragged = len(set(new.tolist())) > 1
    size = np.exp(rng.normal(size=(int(new.sum()), 1, 1)) * 2)       # some scales grow by a lot
    (k, k64), (v, v64) = (bf16(size * rng.standard_normal((int(new.sum()), hkv, D))) for _ in "kv")
    kd, wide = strided(k, 4 if packed else 0)
    vd, _ = strided(v, 4 if packed else 0)
    step, cu = step_of(dev, new, 6, ragged, kv_stride_t=wide.shape[1] * D)
    S.shplb_cache_append(dev.cache, step, kd, vd, stream())
    torch.cuda.synchronize()
    orc.append(c, k64, v64, cu)
    dev.check_same(c)
    S.shplb_cache_append(dev.cache, step, kd, vd, stream())          # again: nothing changes
    dev.check_same(c)
    # all that is held, the last token of every head in the sequence's last row, three rows behind the last sequence
    total = int(lens.sum())
    back = torch.full((total + 3, hkv + 2, D), 5.0, dtype=torch.bfloat16, device=DEV)
    want = [np.full((total + 3, hkv, D), 5.0) for _ in "kv"]
    kb, vb = back[:, 1:1 + hkv], torch.full((total + 3, hkv + 2, D), 5.0, dtype=torch.bfloat16, device=DEV)[:, 1:1 + hkv]
    step, cu = step_of(dev, lens, 6, True, kv_stride_t=(hkv + 2) * D, behind=3)
    S.shplb_cache_load(dev.cache, step, kb, vb, stream())
    orc.load(c, *want, cu)
    np.testing.assert_array_equal(kb.double().cpu().numpy(), want[0])
    np.testing.assert_array_equal(vb.double().cpu().numpy(), want[1])
    assert (back[:, 0] == 5).all() and (back[:, -1] == 5).all()


@FORMATS
def test_append_token_after_token(fmt):
    # forty tokens one by one, now larger, now smaller, through the end of a page
    rng = np.random.default_rng(fmt)
    c = state(rng, [[100, 40]], 64, fmt, spare=2)
    (k0, k64), (v0, v64) = (bf16(rng.standard_normal((100, 2, D))) for _ in "kv")
    dev = Device(c)
    step, cu = step_of(dev, [100], 4, False)
    S.shplb_cache_append(dev.cache, step, k0.to(DEV), v0.to(DEV), stream())
    orc.append(c, k64, v64, cu)
    step, cu = step_of(dev, [1], 4, False)
    for t in range(40):
        size = [0.1, 1, 3, 2, 30][t % 5] * (1 + t / 10)
        (k, k64), (v, v64) = (bf16(size * rng.standard_normal((1, 2, D))) for _ in "kv")
        c.lens += 1
        dev.lens += 1
        S.shplb_cache_append(dev.cache, step, k.to(DEV), v.to(DEV), stream())
        orc.append(c, k64, v64, cu)
        dev.check_same(c)


@FORMATS
def test_append_of_extreme_values(fmt):
    # zeros, the smallest and the largest bf16 numbers, values at the border between two scales, and one that is not finite
    rng = np.random.default_rng(11)
    border = orc.LARGEST[fmt] * 2.0 ** -5
    sizes = [0.0, 1e-38, 9.2e-41, 3.3e38, border, border * (1 + 2.0 ** -7), 1.0, 1.0]
    c = state(rng, [[20]] * len(sizes), 64, fmt)
    x = rng.uniform(-1, 1, size=(len(sizes), 20, 1, D))
    x[:, 3, 0, 5] = 1.0
    x *= np.array(sizes)[:, None, None, None]
    x[6, 7, 0, 9], x[7, 1, 0, 0] = np.inf, np.nan
    k, k64 = bf16(x.reshape(-1, 1, D))
    v, v64 = bf16(-x.reshape(-1, 1, D))
    dev = Device(c)
    step, cu = step_of(dev, [20] * len(sizes), 1, False)
    S.shplb_cache_append(dev.cache, step, k.to(DEV), v.to(DEV), stream())
    orc.append(c, k64, v64, cu)
    dev.check_same(c)
    # finite tokens that follow do not mend the page; one that is not finite takes the others of its page along
    c.lens += 1
    dev.lens += 1
    k, k64 = bf16(np.where(np.arange(len(sizes)) == 4, np.nan, 1.0)[:, None, None] * np.ones((1, 1, D)))
    step, cu = step_of(dev, [1] * len(sizes), 1, False)
    S.shplb_cache_append(dev.cache, step, k.to(DEV), k.to(DEV), stream())
    orc.append(c, k64, k64, cu)
    dev.check_same(c)
    out = torch.zeros((len(sizes) * 21, 1, D), dtype=torch.bfloat16, device=DEV)
    out2 = torch.zeros_like(out)
    step, cu = step_of(dev, [21] * len(sizes), 1, False)
    S.shplb_cache_load(dev.cache, step, out, out2, stream())
    got = out.double().cpu().numpy().reshape(len(sizes), 21, D)
    assert np.isnan(got[[4, 6, 7]]).all() and np.isfinite(got[[0, 1, 2, 3, 5]]).all()


# ---- attention ----------------------------------------------------------------------------------------------------------

ATTNS = {
    # tokens held per sequence, new ones, query heads, KV heads
    "one_token": ([1], [1], 4, 1),
    "short": ([777], [1], 32, 8),
    "ragged": ([1, 0, 63, 64, 65, 127, 128, 129, 1000, 301], [1] * 10, 8, 2),
    "mha": ([300, 77], [1, 1], 3, 3),
    "one_kv_head": ([500], [1], 16, 1),
    "some_without": ([300, 20, 0, 200], [2, 0, 3, 5], 8, 2),
    "sees_nothing": ([2, 5, 130], [5, 5, 5], 4, 2),
    "rows_17": ([400], [17], 2, 2),
    "rows_32": ([333, 90], [8, 8], 8, 2),
    "rows_60": ([333, 90], [15, 3], 8, 2),
    "rows_200": ([333, 90, 700], [50, 1, 37], 8, 2),
    "prompt": ([260], [260], 4, 2),
}


def run_attn(c, q, cu, dev, step, weight_in=None, packed=0):
    qd, wide = strided(q, packed)
    out = torch.full_like(wide, 9.0)
    lse = torch.full((q.shape[1], step.c.n_tokens), 9.0, device=DEV)
    ws = attn_workspace(dev, step)
    w_out = None
    if weight_in is not None:
        w_out = torch.full(weight_in.shape, 9.0, device=DEV)
        weight_in = torch.from_numpy(weight_in).to(DEV)
    lo = packed // 2
    S.shplb_cache_attn(dev.cache, step, qd, out[:, lo:lo + q.shape[1]], lse, weight_in, w_out, ws, stream())
    torch.cuda.synchronize()
    n = int(cu[-1])
    assert (out[n:] == 9).all() and (lse[:, n:] == 9).all()          # rows behind the last sequence
    if packed:
        assert (out[:, :lo] == 9).all() and (out[:, lo + q.shape[1]:] == 9).all()
    got = out[:, lo:lo + q.shape[1]].double().cpu().numpy(), lse.double().cpu().numpy()
    return got + (None if w_out is None else w_out.double().cpu().numpy(),)


@FORMATS
@BLOCKS
@pytest.mark.parametrize("room", [0, 4096], ids=["short", "long"])
@pytest.mark.parametrize("name", ATTNS)
def test_attn(name, room, block, fmt):
    # room: tokens that the page table has places for; a cache of many is worked on by shares of all heads' keys, one of few head by head
    lens, new, hq, hkv = ATTNS[name]
    print("case", name, room, block, fmt, flush=True)
    rng = np.random.default_rng([block, fmt, len(name)])
    lens = np.repeat(np.array(lens)[:, None], hkv, 1)
    if name in ("ragged", "rows_60"):                    # heads of lengths of their own
        lens = np.maximum(np.minimum(lens, 1), (lens * rng.uniform(0.3, 1, size=lens.shape)).astype(int))
    c = filled(rng, lens, block, fmt, max_pages=room // block or None)
    ragged = len(set(new)) > 1
    behind = 2 if ragged else 0
    q, q64 = bf16(2 * rng.standard_normal((sum(new) + behind, hq, D)))
    dev = Device(c)
    packed = 6 if name in ("short", "rows_60", "mha") else 0
    step, cu = step_of(dev, new, hq, ragged, **(dict(behind=behind) if ragged else {}), q_stride_t=(hq + packed) * D)
    kv_of = [h // (hq // hkv) for h in range(hq)]
    w = rng.random((*lens.shape, c.capacity)).astype(np.float32)
    out, lse, w_out = run_attn(c, q, cu, dev, step, w, packed)
    check_attn(c, out, lse, q64, cu, kv_of, got_weight=w_out, weight_in=w)
    behind_len = np.arange(c.capacity) >= c.lens[..., None]
    assert (w_out[behind_len] == 9).all()
    # without weights and denominators: the same output, bit for bit, also on a second call
    for _ in range(2):
        again, _, _ = run_attn(c, q, cu, dev, step, None, packed)
        np.testing.assert_array_equal(again, out)
    dev.check_same(c)                                    # it only reads


@FORMATS
def test_attn_long_heads_in_many_pieces(fmt):
    # two heads of 40000 and 25 tokens, far more pieces than items, and of 64 rows of which some are of another tile
    rng = np.random.default_rng(5)
    c = filled(rng, [[40000, 25]], 128, fmt)
    dev = Device(c)
    for n in (1, 20):
        q, q64 = bf16(2 * rng.standard_normal((n, 8, D)))
        step, cu = step_of(dev, [n], 8, False)
        w = np.zeros((1, 2, c.capacity), np.float32)
        out, lse, w_out = run_attn(c, q, cu, dev, step, w)
        check_attn(c, out, lse, q64, cu, [h // 4 for h in range(8)], got_weight=w_out, weight_in=w)


def test_attn_many_short_sequences():
    # 700 sequences x 6 heads: every workgroup has several items, and finds them behind hundreds of others
    rng = np.random.default_rng(6)
    lens = rng.integers(0, 90, size=(700, 6))
    new = rng.integers(0, 3, size=700)
    c = filled(rng, lens, 64, orc.E4M3)
    q, q64 = bf16(rng.standard_normal((int(new.sum()), 12, D)))
    dev = Device(c)
    step, cu = step_of(dev, new, 12, True)
    w = rng.random((700, 6, c.capacity)).astype(np.float32)
    out, lse, w_out = run_attn(c, q, cu, dev, step, w)
    check_attn(c, out, lse, q64, cu, [h // 2 for h in range(12)], got_weight=w_out, weight_in=w)


@FORMATS
@pytest.mark.parametrize("tokens", [1, 5, 9, 17, 33, 80])
@pytest.mark.parametrize("room", [None, 64])
def test_attn_weights_in_place(room, tokens, fmt):
    # added to where they come from, bit for bit what goes elsewhere: 4 to 320 rows, those behind the 128th added to what the others left
    rng = np.random.default_rng([tokens, fmt])
    c = filled(rng, [[700, 321], [130, 1025]], 64, fmt, max_pages=room)
    q, q64 = bf16(rng.standard_normal((2 * tokens, 8, D)))
    dev = Device(c)
    step, cu = step_of(dev, [tokens] * 2, 8, False)
    w = rng.random((2, 2, c.capacity)).astype(np.float32)
    out, lse, elsewhere = run_attn(c, q, cu, dev, step, w)
    check_attn(c, out, lse, q64, cu, [h // 4 for h in range(8)], got_weight=elsewhere, weight_in=w)
    here = torch.from_numpy(w).to(DEV)
    o = torch.empty((2 * tokens, 8, D), dtype=torch.bfloat16, device=DEV)
    for _ in range(3):
        here.copy_(torch.from_numpy(w))
        S.shplb_cache_attn(dev.cache, step, q.to(DEV), o, None, here, here, attn_workspace(dev, step), stream())
        there = np.arange(c.capacity) < c.lens[..., None]
        np.testing.assert_array_equal(here.double().cpu().numpy()[there], elsewhere[there])
        np.testing.assert_array_equal(here.cpu().numpy()[~there], w[~there])
        np.testing.assert_array_equal(o.double().cpu().numpy(), out)


@FORMATS
@pytest.mark.parametrize("tokens,room", [(2, None), (11, None), (11, 80)])
def test_attn_few_of_many_sequences(tokens, room, fmt):
    # 700 sequences of which seven have tokens in this step, the first and the last among them, and a KV head without query heads
    rng = np.random.default_rng([tokens, fmt])
    new = np.zeros(700, int)
    new[[0, 1, 63, 64, 65, 400, 699]] = tokens
    lens = rng.integers(0, 150, size=(700, 3))
    c = filled(rng, lens, 64, fmt, max_pages=room)
    kv_of = [2, 0, 2]
    q, q64 = bf16(rng.standard_normal((int(new.sum()), 3, D)))
    dev = Device(c)
    step, cu = step_of(dev, new, 3, True, kv_head_of=kv_of)
    w = rng.random((700, 3, c.capacity)).astype(np.float32)
    out, lse, w_out = run_attn(c, q, cu, dev, step, w)
    check_attn(c, out, lse, q64, cu, kv_of, got_weight=w_out, weight_in=w)


@FORMATS
@pytest.mark.parametrize("room", [1, 64], ids=["short", "long"])
def test_attn_one_token_of_every_scale(room, fmt):
    # a head of one token: its output is that token's value, whatever the page's scale is.  (The probability is within 2^-20 of one, and the value a bf16
    # number: half a step, 2^-9 of it, away from rounding to another.)
    rng = np.random.default_rng(fmt)
    scales = 2.0 ** np.arange(-110, 101)
    c = state(rng, np.ones((scales.size, 1), int), 64, fmt, spare=0, max_pages=room)
    c.k_scale[:] = 2.0 ** -6
    c.k_pages[:] = orc.encode(rng.standard_normal(c.k_pages.shape), fmt)
    most = orc.LARGEST[fmt]
    c.v_pages[c.table[:, 0, 0], 0] = orc.encode(rng.uniform(-most, most, size=(scales.size, D)), fmt)
    c.v_scale[c.table[:, 0, 0]] = scales
    q, _ = bf16(rng.standard_normal((scales.size, 2, D)))
    dev = Device(c)
    step, cu = step_of(dev, np.ones(scales.size, int), 2, False)
    w = np.zeros((scales.size, 1, c.capacity), np.float32)
    out, _, w_out = run_attn(c, q, cu, dev, step, w)
    want = np.stack([c.values("v", s, 0, 1)[0] for s in range(scales.size)])
    np.testing.assert_array_equal(out, np.stack([want, want], 1))
    assert (np.abs(w_out[:, 0, 0] - 2) <= 2 * 2.0 ** -20).all()


@FORMATS
@pytest.mark.parametrize("tokens", [1, 6])
def test_attn_more_heads_than_compute_units(tokens, fmt):
    # 110 sequences x 4 heads in short caches: a head a workgroup, or a tile of one, whatever finds a place first
    rng = np.random.default_rng([tokens, fmt])
    lens = np.maximum(rng.integers(0, 300, size=(110, 4)), np.where(np.arange(110) == 50, 1900, 0)[:, None])
    c = filled(rng, lens, 128, fmt)
    q, q64 = bf16(rng.standard_normal((110 * tokens, 16, D)))
    dev = Device(c)
    step, cu = step_of(dev, [tokens] * 110, 16, False)
    w = rng.random((110, 4, c.capacity)).astype(np.float32)
    out, lse, w_out = run_attn(c, q, cu, dev, step, w)
    check_attn(c, out, lse, q64, cu, [h // 4 for h in range(16)], got_weight=w_out, weight_in=w)


@pytest.mark.parametrize("room", [None, 64])
def test_attn_mapped_heads_and_scale(room):
    rng = np.random.default_rng(7)
    kv_of = [2, 0, 2, 2, 0, 2]                           # the second KV head has no query head
    c = filled(rng, [[200, 150, 330], [64, 1, 0]], 64, orc.INT8, max_pages=room)
    q, q64 = bf16(rng.standard_normal((4, 6, D)))
    dev = Device(c)
    step, cu = step_of(dev, [2, 2], 6, False, kv_head_of=kv_of, softmax_scale=0.03)
    w = rng.random((2, 3, c.capacity)).astype(np.float32)
    out, lse, w_out = run_attn(c, q, cu, dev, step, w)
    check_attn(c, out, lse, q64, cu, kv_of, scale=float(np.float32(0.03)), got_weight=w_out, weight_in=w)


@FORMATS
@pytest.mark.parametrize("room", [None, 64])
def test_attn_of_extreme_sizes(room, fmt):
    # queries and keys of very different size: scales far apart, scores near 0 and in the hundreds, values of 1e30 beside 1e-30
    rng = np.random.default_rng(8)
    c = state(rng, [[200]] * 4, 64, fmt, max_pages=room)
    sizes = np.array([1e-30, 1e-3, 1.0, 1e3])
    k, k64 = bf16((sizes[:, None, None, None] * rng.standard_normal((4, 200, 1, D))).reshape(-1, 1, D))
    per_page = np.exp(rng.uniform(-60, 60, size=(4, 4)))[:, np.arange(200) // 64]
    v, v64 = bf16((per_page[..., None, None] * rng.standard_normal((4, 200, 1, D))).reshape(-1, 1, D))
    orc.append(c, k64, v64, np.arange(5) * 200)
    q, q64 = bf16((np.array([1e25, 1e3, 10.0, 3e-4])[:, None, None] * rng.standard_normal((4, 4, D))))
    dev = Device(c)
    step, cu = step_of(dev, [1] * 4, 4, False)
    out, lse, _ = run_attn(c, q, cu, dev, step)
    check_attn(c, out, lse, q64, cu, [0] * 4)


@pytest.mark.parametrize("room", [None, 64])
def test_attn_nothing_to_do(room):
    # a step without a token: nothing but the weights, which are copied
    rng = np.random.default_rng(9)
    c = filled(rng, [[100, 64], [0, 3]], 64, orc.E4M3, max_pages=room)
    dev = Device(c)
    step = S.Step(2, 4, 2, 0, 0)
    w = torch.rand((2, 2, c.capacity), device=DEV)
    w_out = torch.full_like(w, 9.0)
    ws = attn_workspace(dev, step)
    S.shplb_cache_attn(dev.cache, step, None, None, None, w, w_out, ws, stream())
    here = torch.arange(c.capacity, device=DEV) < dev.lens[..., None]
    assert torch.equal(w_out, torch.where(here, w, 9.0))
    # weights in place, from none
    step = S.Step(2, 4, 2)
    q = torch.randn((2, 4, D), device=DEV).to(torch.bfloat16)
    out, first = torch.empty_like(q), torch.zeros_like(w)
    S.shplb_cache_attn(dev.cache, step, q, out, None, None, first, attn_workspace(dev, step), stream())
    twice = first.clone()
    S.shplb_cache_attn(dev.cache, step, q, out, None, twice, twice, attn_workspace(dev, step), stream())
    assert torch.equal(twice, first + first)
    np.testing.assert_allclose(first.sum(2).cpu().numpy(), [[2, 2], [0, 2]], rtol=1e-5)


# ---- eviction -----------------------------------------------------------------------------------------------------------


def evict_case(rng, lens, keep, sink, recent, block, to_block, fmt, to_pages, kind="heavy"):
    c = filled(rng, lens, block, fmt)
    lens = c.lens
    w = np.exp(2 * rng.standard_normal((*lens.shape, c.capacity))).astype(np.float32)
    if kind == "ties":                                   # few distinct values, zeros of both signs, NaN, infinities, negative ones
        w = rng.choice(np.array([0.0, -0.0, 1.0, 2.0, np.nan, np.inf, -1.0, -np.inf, 1e-42], np.float32), size=w.shape)
    if kind == "zeros":
        w[:] = 0
    keep = np.broadcast_to(np.asarray(keep, np.int32), lens.shape)
    to = state(rng, np.full(lens.shape, to_pages * to_block), to_block, fmt, spare=0)
    dev, dto = Device(c), Device(to)
    wd, kd = torch.from_numpy(w).to(DEV), torch.from_numpy(keep.copy()).to(DEV)
    w_out = torch.zeros((*lens.shape, to.capacity), device=DEV)
    kept = torch.zeros((*lens.shape, to.capacity), dtype=torch.int32, device=DEV)
    ws = torch.empty(S.shplb_cache_evict_workspace_bytes(dev.cache), dtype=torch.uint8, device=DEV).fill_(0xff)
    for _ in range(2):                                   # twice: the workspace needs no clearing, results are the same
        S.shplb_cache_evict(dev.cache, wd, kd, sink, recent, dto.cache, w_out, kept, ws, stream())
    torch.cuda.synchronize()
    want_w, want_kept = orc.evict(c, w, keep, sink, recent, to)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    np.testing.assert_array_equal(w_out.cpu().numpy(), want_w)
    dto.check_same(to)
    dev.check_same(c)


@FORMATS
@pytest.mark.parametrize("kind", ["heavy", "ties", "zeros"])
@pytest.mark.parametrize("blocks", [(128, 128), (64, 128), (128, 64)])
def test_evict(kind, blocks, fmt):
    rng = np.random.default_rng([fmt, len(kind), blocks[1]])
    lens = rng.integers(0, 500, size=(6, 3))
    lens[0, 0], lens[1, 1], lens[2, 2] = 0, 1, 499
    keep = rng.integers(0, 300, size=(6, 3))
    keep[0], keep[3, 0], keep[4, 0] = 1000, 0, -5
    evict_case(rng, lens, keep, 5, 9, *blocks, fmt, 512 // blocks[1], kind)


@pytest.mark.parametrize("sink,recent", [(0, 0), (0, 3), (70, 0), (400, 400), (1, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_evict_sinks_and_recents(sink, recent):
    # ... where those alone are more than the head holds, and more than there is room for (two pages of 64)
    rng = np.random.default_rng(3)
    evict_case(rng, [[300, 40], [128, 129]], [[0, 100], [3, 64]], sink, recent, 64, 64, orc.E4M3, 2)


def test_evict_long_head():
    rng = np.random.default_rng(4)
    evict_case(rng, [[70001, 2000, 64]], [[9000, 1999, 1]], 128, 128, 128, 128, orc.INT8, 80)
    evict_case(rng, [[70001, 2000, 64]], [[9000, 1999, 1]], 128, 128, 128, 128, orc.E4M3, 80, "ties")


# tokens of three heads: where one workgroup sees all of a head's weights, and where parts of 8192 are counted by themselves
EVICTS = {"one_part": [5000, 8000, 2049], "whole_part": [8064, 3, 8000], "twice_that": [12001, 16256, 8193],
          "parts": [16385, 8193, 8192], "last_of_a_part": [24448, 16384, 0]}


@pytest.mark.parametrize("kind", ["heavy", "ties", "zeros"])
@pytest.mark.parametrize("sink,recent", [(3, 40), (8200, 150), (100, 8200)])
@pytest.mark.parametrize("name", EVICTS)
def test_evict_parts(name, sink, recent, kind):
    rng = np.random.default_rng([len(name), sink, len(kind)])
    evict_case(rng, [EVICTS[name]], [[1500, 8300, 8192]], sink, recent, 128, 64, orc.E4M3, 150, kind)


def test_evict_inside_one_pool():
    rng = np.random.default_rng(14)
    c = filled(rng, [[200, 130]], 64, orc.E4M3, spare=0, extra_pages=6)
    to = c.copy()
    free = sorted(set(range(c.n_pages)) - set(c.table[c.table >= 0].tolist()))
    to.table = np.array(free[:6], np.int32).reshape(1, 2, 3)
    to.k_pages, to.v_pages, to.k_scale, to.v_scale = c.k_pages, c.v_pages, c.k_scale, c.v_scale      # one pool
    to.lens = np.zeros((1, 2), np.int32)
    dev = Device(c)
    dto = S.Cache(dev.k_pages, dev.v_pages, dev.k_scale, dev.v_scale, (tt := torch.from_numpy(to.table).to(DEV)),
                  (tl := torch.zeros((1, 2), dtype=torch.int32, device=DEV)), 1, 2, 64, 3, c.n_pages)
    w = rng.random((1, 2, c.capacity)).astype(np.float32)
    w_out = torch.zeros((1, 2, 192), device=DEV)
    kept = torch.zeros((1, 2, 192), dtype=torch.int32, device=DEV)
    ws = torch.empty(S.shplb_cache_evict_workspace_bytes(dev.cache), dtype=torch.uint8, device=DEV)
    S.shplb_cache_evict(dev.cache, torch.from_numpy(w).to(DEV), torch.tensor([[70, 130]], dtype=torch.int32, device=DEV), 1, 2, dto,
                        w_out, kept, ws, stream())
    orc.evict(c, w, np.array([[70, 130]]), 1, 2, to)
    dev.check_same(c)
    assert tl.tolist() == to.lens.tolist() == [[70, 130]] and tt is not None


# ---- what should not happen, and what else a program does ---------------------------------------------------------------


@pytest.mark.parametrize("room", [None, 64])
def test_damaged_pages_lengths_and_offsets(room):
    # pages outside the pool, lengths outside the table, offsets outside the rows: nothing is touched outside, results say NaN
    rng = np.random.default_rng(21)
    c = filled(rng, [[200, 200], [200, 200], [90, 90]], 64, orc.E4M3, max_pages=room)
    c.table[0, 0, 1], c.table[0, 1, 0], c.table[1, 0, 3] = -7, c.n_pages, 2 ** 31 - 1
    c.lens[1, 1], c.lens[2, 0] = c.capacity + 1, -1
    dev = Device(c)
    q, q64 = bf16(rng.standard_normal((3, 4, D)))
    step, cu = step_of(dev, [1] * 3, 4, False)
    w = rng.random((3, 2, c.capacity)).astype(np.float32)
    out, lse, w_out = run_attn(c, q, cu, dev, step, w)
    check_attn(c, out, lse, q64, cu, [0, 0, 1, 1], got_weight=w_out, weight_in=w)
    assert np.isnan(out[0]).all() and np.isnan(out[1]).all() and np.isnan(out[2, :2]).all() and np.isfinite(out[2, 2:]).all()
    k, k64 = bf16(rng.standard_normal((3, 2, D)))
    S.shplb_cache_append(dev.cache, step, k.to(DEV), k.to(DEV), stream())
    orc.append(c, k64, k64, cu)
    dev.check_same(c)
    back = torch.full((300, 2, D), 5.0, dtype=torch.bfloat16, device=DEV)
    back2, want = back.clone(), [np.full((300, 2, D), 5.0) for _ in "kv"]
    step, cu = step_of(dev, [100] * 3, 4, False)
    S.shplb_cache_load(dev.cache, step, back, back2, stream())
    orc.load(c, *want, cu)
    np.testing.assert_array_equal(back.double().cpu().numpy(), want[0])
    to = state(rng, np.full((3, 2), 128), 64, orc.E4M3, spare=0)
    to.table[2, 1, 0] = -1
    dto = Device(to)
    w_out = torch.zeros((3, 2, 128), device=DEV)
    kept = torch.zeros((3, 2, 128), dtype=torch.int32, device=DEV)
    ws = torch.empty(S.shplb_cache_evict_workspace_bytes(dev.cache), dtype=torch.uint8, device=DEV)
    S.shplb_cache_evict(dev.cache, torch.from_numpy(w).to(DEV), torch.full((3, 2), 100, dtype=torch.int32, device=DEV), 1, 1, dto.cache,
                        w_out, kept, ws, stream())
    _, want_kept = orc.evict(c, w, np.full((3, 2), 100), 1, 1, to)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    dto.check_same(to)
    # rows that cu_tokens leaves outside: below 0, behind the last, backwards
    bad = torch.tensor([-5, 2, 1, 90], dtype=torch.int32, device=DEV)
    step = S.Step(3, 4, 2, 3, 2, bad)
    o = torch.full((3, 4, D), 9.0, dtype=torch.bfloat16, device=DEV)
    S.shplb_cache_attn(dev.cache, step, q.to(DEV), o, None, None, None, attn_workspace(dev, step), stream())
    torch.cuda.synchronize()


@FORMATS
@pytest.mark.parametrize("which", ["k", "v", "number"])
@pytest.mark.parametrize("hq,tokens", [(1, 5), (8, 5), (8, 20)])
@pytest.mark.parametrize("room", [None, 64])
def test_rows_that_see_nothing_of_a_damaged_page(room, hq, tokens, which, fmt):
    # the last page has no scale, or is none: rows that see none of it are as if it were not there, their weights, too, whatever the pool's first
    # page holds
    rng = np.random.default_rng([hq, tokens])
    c = filled(rng, [[130], [64 + 2]], 64, fmt, max_pages=room)
    free = sorted(set(range(c.n_pages)) - set(c.table[c.table >= 0].tolist()))[-1]
    for pages, scale in ((c.k_pages, c.k_scale), (c.v_pages, c.v_scale)):
        pages[free], scale[free] = pages[0], scale[0]
        pages[0] = 0x7f
    c.table[c.table == 0] = free
    for s, i in ((0, 2), (1, 1)):
        if which == "number":
            c.table[s, 0, i] = c.n_pages
        else:
            (c.k_scale if which == "k" else c.v_scale)[c.table[s, 0, i]] = np.nan
    dev = Device(c)
    q, q64 = bf16(rng.standard_normal((2 * tokens, hq, D)))
    step, cu = step_of(dev, [tokens] * 2, hq, False)
    w = rng.random((2, 1, c.capacity)).astype(np.float32)
    out, lse, w_out = run_attn(c, q, cu, dev, step, w)
    check_attn(c, out, lse, q64, cu, [0] * hq, got_weight=w_out, weight_in=w)
    seen = np.array([tokens - 2, tokens - 1, 2 * tokens - 2, 2 * tokens - 1])
    assert np.isnan(out[seen]).all() and np.isfinite(np.delete(out, seen, 0)).all()


@FORMATS
@pytest.mark.parametrize("tokens", [3, 20])
@pytest.mark.parametrize("room", [None, 64])
def test_queries_that_are_not_finite(room, tokens, fmt):
    # an infinity that meets keys of both signs, of one sign, or none at all, and a NaN: what it reaches is NaN, the other rows are as they are
    rng = np.random.default_rng([tokens, fmt])
    lens = np.array([[150], [400], [tokens - 2], [200]])
    c = state(rng, lens, 64, fmt, max_pages=room)
    cu = np.concatenate([[0], np.cumsum(lens[:, 0])])
    (k, _), (v, v64) = (bf16(rng.standard_normal((int(cu[-1]), 1, D))) for _ in "kv")
    k[:, 0, 7] = -k[:, 0, 7].abs() - 0.5                 # never zero, always negative
    orc.append(c, k.double().numpy(), v64, cu)
    q, _ = bf16(rng.standard_normal((4 * tokens, 4, D)))
    q[1, 0, 7], q[2, 3, 7], q[2, 2, 9] = np.inf, -np.inf, np.inf
    q[2 * tokens + 1, 0, 7] = np.inf                     # sees nothing
    q[3 * tokens, 1, 0] = np.nan
    dev = Device(c)
    step, cu = step_of(dev, [tokens] * 4, 4, False)
    w = np.zeros((4, 1, c.capacity), np.float32)
    with np.errstate(invalid="ignore"):
        out, lse, w_out = run_attn(c, q, cu, dev, step, w)
        check_attn(c, out, lse, q.double().numpy(), cu, [0] * 4, got_weight=w_out, weight_in=w)
    bad = np.isnan(out).all(2)
    assert bad.sum() == 4 and bad[1, 0] and bad[2, 3] and bad[2, 2] and bad[3 * tokens, 1] and not np.isnan(out[~bad]).any()
    assert (out[2 * tokens + 1] == 0).all() and np.isneginf(lse[:, 2 * tokens + 1]).all()


@FORMATS
def test_heads_apart(fmt):
    # heads further from one another than their 128 dims, rows further than their heads, at addresses of 16 bytes
    rng = np.random.default_rng([26, fmt])
    hq, hkv, n, far = 4, 2, 5, 152
    apart = lambda heads: (torch.full((3 * n * (heads + 1) * far + 8,), 9.0, dtype=torch.bfloat16, device=DEV)[8:]
                           .view(3 * n, heads + 1, far)[:, :heads, :D])
    c = filled(rng, [[100, 30], [n, 64], [300, 299]], 64, fmt, spare=1)
    dev = Device(c)
    (k, k64), (v, v64) = (bf16(rng.standard_normal((3 * n, hkv, D))) for _ in "kv")
    q, q64 = bf16(rng.standard_normal((3 * n, hq, D)))
    kd, vd, qd, od, bk, bv = (apart(x) for x in (hkv, hkv, hq, hq, hkv, hkv))
    kd.copy_(k), vd.copy_(v), qd.copy_(q)
    step, cu = step_of(dev, [n] * 3, hq, False, q_stride_h=far, q_stride_t=(hq + 1) * far, kv_stride_h=far, kv_stride_t=(hkv + 1) * far)
    S.shplb_cache_append(dev.cache, step, kd, vd, stream())
    orc.append(c, k64, v64, cu)
    dev.check_same(c)
    S.shplb_cache_load(dev.cache, step, bk, bv, stream())
    want = [np.full((3 * n, hkv, D), 9.0) for _ in "kv"]
    orc.load(c, *want, cu)
    np.testing.assert_array_equal(bk.double().cpu().numpy(), want[0])
    np.testing.assert_array_equal(bv.double().cpu().numpy(), want[1])
    S.shplb_cache_attn(dev.cache, step, qd, od, None, None, None, attn_workspace(dev, step), stream())
    check_attn(c, od.double().cpu().numpy(), None, q64, cu, [0, 0, 1, 1])
    for x, heads in ((od, hq), (bk, hkv)):               # what lies between the heads is as it was
        whole = torch.as_strided(x, (3 * n, heads + 1, far), ((heads + 1) * far, far, 1))
        assert (whole[:, :, D:] == 9).all() and (whole[:, heads] == 9).all()


def test_pages_far_into_a_pool():
    # byte offsets beyond 32 bits: a pool of 4.9 GB of keys and as much of values, of which the last pages are used
    n_pages = 300000
    rng = np.random.default_rng(22)
    c = filled(rng, [[300, 200]], 128, orc.E4M3, extra_pages=0, spare=0)
    k_pages = torch.empty((n_pages, 128, D), dtype=torch.uint8, device=DEV)
    v_pages = torch.empty_like(k_pages)
    k_scale, v_scale = torch.ones(n_pages, device=DEV), torch.ones(n_pages, device=DEV)
    at = n_pages - c.n_pages
    small = Device(c)
    for big, mine in ((k_pages, small.k_pages), (v_pages, small.v_pages), (k_scale, small.k_scale), (v_scale, small.v_scale)):
        big[at:] = mine
    table = torch.where(small.table >= 0, small.table + at, small.table).contiguous()
    cache = S.Cache(k_pages, v_pages, k_scale, v_scale, table, small.lens, 1, 2, 128, small.max_pages, n_pages)
    q, q64 = bf16(rng.standard_normal((1, 4, D)))
    step, cu = step_of(small, [1], 4, False)
    out = torch.empty((1, 4, D), dtype=torch.bfloat16, device=DEV)
    k, k64 = bf16(rng.standard_normal((1, 2, D)))
    S.shplb_cache_append(cache, step, k.to(DEV), k.to(DEV), stream())
    S.shplb_cache_attn(cache, step, q.to(DEV), out, None, None, None, attn_workspace(small, step), stream())
    orc.append(c, k64, k64, cu)
    check_attn(c, out.double().cpu().numpy(), None, q64, cu, [0, 0, 1, 1])
    back, back2 = (torch.zeros((300, 2, D), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    step, cu = step_of(small, [300], 4, False)
    S.shplb_cache_load(cache, step, back, back2, stream())
    want = [np.zeros((300, 2, D)) for _ in "kv"]
    orc.load(c, *want, cu)
    np.testing.assert_array_equal(back2.double().cpu().numpy(), want[1])


@pytest.mark.parametrize("room", [None, 40])
def test_shared_pages_and_another_stream(room):
    # three sequences read one prefix; on a stream that is not the current one
    rng = np.random.default_rng(23)
    c = filled(rng, [[256 + 10, 256 + 10]] * 3, 128, orc.INT8, max_pages=room)
    c.table[1:, :, :2] = c.table[0, :, :2]
    q, q64 = bf16(rng.standard_normal((3, 8, D)))
    dev = Device(c)
    step, cu = step_of(dev, [1] * 3, 8, False)
    qd, out, ws = q.to(DEV), torch.empty((3, 8, D), dtype=torch.bfloat16, device=DEV), attn_workspace(dev, step)
    w = torch.zeros((3, 2, c.capacity), device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(stream())
    S.shplb_cache_attn(dev.cache, step, qd, out, None, None, w, ws, side)
    side.synchronize()
    check_attn(c, out.double().cpu().numpy(), None, q64, cu, [h // 4 for h in range(8)], got_weight=w.double().cpu().numpy(),
               weight_in=np.zeros(w.shape, np.float32))


@pytest.mark.parametrize("room", [None, 40])
def test_decoding_step_in_a_hip_graph(room):
    # one token of three sequences appended and attended to, captured once and replayed while lengths and inputs change; with eager
    # calls and other use of the workspace in between
    rng = np.random.default_rng(24)
    c = filled(rng, [[60, 60], [130, 90], [1, 2]], 64, orc.E4M3, **(dict(spare=2) if room is None else dict(max_pages=room, spare=2)))
    dev = Device(c)
    hq = 8
    step, cu = step_of(dev, [1] * 3, hq, False)
    k, v = (torch.zeros((3, 2, D), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    q = torch.zeros((3, hq, D), dtype=torch.bfloat16, device=DEV)
    out, lse, w = torch.zeros_like(q), torch.zeros((hq, 3), device=DEV), torch.zeros((3, 2, c.capacity), device=DEV)
    ws = attn_workspace(dev, step)
    side = torch.cuda.Stream()
    side.wait_stream(stream())
    graph = torch.cuda.CUDAGraph()

    def both(st):
        S.shplb_cache_append(dev.cache, step, k, v, st)
        S.shplb_cache_attn(dev.cache, step, q, out, lse, w, w, ws, st)

    with torch.cuda.stream(side):
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            both(side)
    torch.cuda.synchronize()
    w64 = np.zeros(w.shape)
    for t in range(8):
        (kt, k64), (vt, v64) = (bf16((1 + t) * rng.standard_normal((3, 2, D))) for _ in "kv")
        qt, q64 = bf16(rng.standard_normal((3, hq, D)))
        k.copy_(kt), v.copy_(vt), q.copy_(qt)
        dev.lens += 1
        c.lens += 1
        ws.random_(0, 255)
        torch.cuda.synchronize()
        if t == 5:
            both(stream())
        else:
            graph.replay()
        torch.cuda.synchronize()
        orc.append(c, k64, v64, cu)
        dev.check_same(c)
        kv_of = [h // 4 for h in range(hq)]
        check_attn(c, out.double().cpu().numpy(), lse.double().cpu().numpy(), q64, cu, kv_of, got_weight=w.double().cpu().numpy(),
                   weight_in=w64)
        w64 = w.double().cpu().numpy()


@pytest.mark.parametrize("n,length,tokens", [(1, 30000, 1), (3, 700, 40), (300, 65, 1), (1, 9000, 100)])
def test_workspaces_end_where_they_say(n, length, tokens):
    # what lies behind a workspace is as it was
    rng = np.random.default_rng(n)
    c = filled(rng, np.full((n, 2), length), 128, orc.E4M3, max_pages=300)
    dev = Device(c)
    step, _ = step_of(dev, [tokens] * n, 8, False)
    q = torch.randn((n * tokens, 8, D), device=DEV).to(torch.bfloat16)
    w = torch.zeros((n, 2, c.capacity), device=DEV)
    to = state(rng, np.full((n, 2), 64), 64, orc.E4M3, spare=0)
    dto = Device(to)
    w_out = torch.zeros((n, 2, to.capacity), device=DEV)
    kept = torch.zeros((n, 2, to.capacity), dtype=torch.int32, device=DEV)
    keep = torch.full((n, 2), 60, dtype=torch.int32, device=DEV)
    for size, call in (
            (S.shplb_cache_attn_workspace_bytes(dev.cache, step),
             lambda ws: S.shplb_cache_attn(dev.cache, step, q, torch.empty_like(q), None, None, w, ws, stream())),
            (S.shplb_cache_evict_workspace_bytes(dev.cache),
             lambda ws: S.shplb_cache_evict(dev.cache, w, keep, 1, 1, dto.cache, w_out, kept, ws, stream()))):
        ws = torch.full((size + (1 << 20),), 0x5a, dtype=torch.uint8, device=DEV)
        call(ws)
        assert (ws[size:] == 0x5a).all()


@FORMATS
def test_two_graphs_of_one_workspace(fmt):
    # a decoding step and a prompt's window with the eviction behind it, captured each, share one workspace and take turns, with the
    # program's own calls in between; every replay leaves what the same calls leave outside of a graph
    rng = np.random.default_rng([25, fmt])
    hq, hkv, n = 8, 2, 9
    c = filled(rng, [[3000, 2500], [400, 900], [64, 1]], 64, fmt, spare=2)
    to = state(rng, np.full((3, hkv), 640), 64, fmt, spare=0)
    dev, dto = Device(c), Device(to)
    one, _ = step_of(dev, [1] * 3, hq, False)
    many, _ = step_of(dev, [n] * 3, hq, False)
    new = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
    k, v, q1, o1 = new(3, hkv, D), new(3, hkv, D), new(3, hq, D), new(3, hq, D)
    q2, o2, back_k, back_v = new(3 * n, hq, D), new(3 * n, hq, D), new(3 * n, hkv, D), new(3 * n, hkv, D)
    w1, w2 = (torch.zeros((3, hkv, c.capacity), device=DEV) for _ in "12")
    lse = torch.zeros((hq, 3 * n), device=DEV)
    keep = torch.full((3, hkv), 500, dtype=torch.int32, device=DEV)
    w_kept = torch.zeros((3, hkv, to.capacity), device=DEV)
    kept = torch.zeros((3, hkv, to.capacity), dtype=torch.int32, device=DEV)
    ws = torch.empty(max(S.shplb_cache_attn_workspace_bytes(dev.cache, one), S.shplb_cache_attn_workspace_bytes(dev.cache, many),
                         S.shplb_cache_evict_workspace_bytes(dev.cache)), dtype=torch.uint8, device=DEV)

    def decode(st):
        S.shplb_cache_append(dev.cache, one, k, v, st)
        S.shplb_cache_attn(dev.cache, one, q1, o1, None, None, w1, ws, st)

    def window(st):
        S.shplb_cache_attn(dev.cache, many, q2, o2, lse, None, w2, ws, st)
        S.shplb_cache_evict(dev.cache, w2, keep, 4, n, dto.cache, w_kept, kept, ws, st)
        S.shplb_cache_load(dev.cache, many, back_k, back_v, st)

    results = [dev.k_pages, dev.v_pages, dev.k_scale, dev.v_scale, o1, w1, o2, lse, w2, dto.k_pages, dto.v_pages, dto.k_scale, dto.v_scale,
               dto.lens, w_kept, kept, back_k, back_v]
    side = torch.cuda.Stream()
    side.wait_stream(stream())
    graphs = []
    for f in (decode, window):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(side):
            torch.cuda.synchronize()
            with torch.cuda.graph(graphs[-1], stream=side):
                f(side)
    torch.cuda.synchronize()
    for t in range(5):
        for x in (k, v, q1, q2):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape))))
        dev.lens += 1
        ws.random_(0, 255)
        before = [x.clone() for x in results]
        torch.cuda.synchronize()
        for g in graphs if t % 2 == 0 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in results]
        for x, y in zip(results, before):                # (the window may have looked at a token that is not there yet)
            x.copy_(y)
        for f in (decode, window) if t % 2 == 0 else (window, decode):
            f(stream())
        torch.cuda.synchronize()
        for x, y in zip(got, results):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_prompt_window_eviction_and_steps():
    """The operators together: a prompt through the sparse prefill and into the cache, its last 32 queries weigh its tokens, every
    head is evicted to its own budget, and decoding goes on behind that."""
    from harness import DevicePass
    from workloads import make_workload
    T, hq, hkv, window = 900, 32, 8, 32
    wl = make_workload(1, seqlens=[T])
    run = DevicePass(wl).run_all()                       # the prompt's own attention
    rng = np.random.default_rng(30)
    c = state(rng, np.full((1, hkv), T), 128, orc.E4M3)
    dev = Device(c)
    step, cu = step_of(dev, [T], hq, False)
    S.shplb_cache_append(dev.cache, step, run.k, run.v, stream())
    orc.append(c, run.k.double().cpu().numpy(), run.v.double().cpu().numpy(), cu)
    kv_of = [h // (hq // hkv) for h in range(hq)]
    step, cu = step_of(dev, [window], hq, False)
    w = torch.zeros((1, hkv, c.capacity), device=DEV)
    out = torch.empty((window, hq, D), dtype=torch.bfloat16, device=DEV)
    S.shplb_cache_attn(dev.cache, step, run.q[T - window:], out, None, None, w, attn_workspace(dev, step), stream())
    check_attn(c, out.double().cpu().numpy(), None, run.q[T - window:].double().cpu().numpy(), cu, kv_of,
               got_weight=w.double().cpu().numpy(), weight_in=np.zeros(w.shape, np.float32))
    keep = rng.integers(100, 600, size=(1, hkv)).astype(np.int32)
    to = state(rng, np.full((1, hkv), 700), 128, orc.E4M3, spare=0)
    dto = Device(to)
    w2 = torch.zeros((1, hkv, to.capacity), device=DEV)
    kept = torch.zeros((1, hkv, to.capacity), dtype=torch.int32, device=DEV)
    ws = torch.empty(S.shplb_cache_evict_workspace_bytes(dev.cache), dtype=torch.uint8, device=DEV)
    S.shplb_cache_evict(dev.cache, w, torch.from_numpy(keep).to(DEV), 16, window, dto.cache, w2, kept, ws, stream())
    want_w, want_kept = orc.evict(c, w.cpu().numpy(), keep, 16, window, to)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    np.testing.assert_array_equal(w2.cpu().numpy(), want_w)
    dto.check_same(to)
    step, cu = step_of(dto, [1], hq, False)
    ws = attn_workspace(dto, step)
    for t in range(3):
        (k, k64), (v, v64) = (bf16(rng.standard_normal((1, hkv, D))) for _ in "kv")
        q, q64 = bf16(rng.standard_normal((1, hq, D)))
        to.lens += 1
        dto.lens += 1
        before = w2.cpu().numpy()
        o = torch.empty((1, hq, D), dtype=torch.bfloat16, device=DEV)
        S.shplb_cache_append(dto.cache, step, k.to(DEV), v.to(DEV), stream())
        S.shplb_cache_attn(dto.cache, step, q.to(DEV), o, None, w2, w2, ws, stream())
        orc.append(to, k64, v64, cu)
        dto.check_same(to)
        check_attn(to, o.double().cpu().numpy(), None, q64, cu, kv_of, got_weight=w2.double().cpu().numpy(), weight_in=before)
