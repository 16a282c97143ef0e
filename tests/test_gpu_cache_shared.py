"""GPU parity of attention behind shared prefixes in the 8-bit cache, through the C ABI against the oracle."""
import numpy as np
import pytest
import torch

import paper_2603_10353_amd as S
from cache_harness import D, DEV, Device, bf16, filled, step_of, strided
from oracle import cache_oracle, window_oracle as orc
from window_harness import check, check_far, far_apart, in_a_large_pool

pytestmark = pytest.mark.gpu
E4M3, INT8 = cache_oracle.E4M3, cache_oracle.INT8
FORMATS = pytest.mark.parametrize("fmt", [E4M3, INT8], ids=["e4m3", "int8"])
HALF, LIFT = 2.0 ** -11, 2.0 ** -32


def stream():
    return torch.cuda.current_stream()


def workspace(pre, dev, step):
    return torch.empty(S.shplb_cache_attn_shared_workspace_bytes(pre.cache, dev.cache, step), dtype=torch.uint8, device=DEV).fill_(0xff)


def cu_of(groups):
    return torch.tensor(groups, dtype=torch.int32, device=DEV)


def call(pre, groups, dev, step, q, ws=None):
    out, lse = torch.full_like(q, 7.0), torch.full((q.shape[1], q.shape[0]), 7.0, device=DEV)
    S.shplb_cache_attn_shared(pre.cache, groups if torch.is_tensor(groups) else cu_of(groups), dev.cache, step, q, out, lse,
                              workspace(pre, dev, step) if ws is None else ws, stream())
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


CASES = {  # lengths of prefixes, cu_prefix, own lengths, new tokens, query heads, KV heads
    "one_sequence": ([[100]], [0, 1], [[5]], [1], 4, 1),
    "one_key": ([[1]], [0, 2], [[1], [2]], [1, 1], 1, 1),
    "samples": ([[300, 200]], [0, 4], [[1, 1], [40, 70], [129, 64], [65, 300]], [1] * 4, 4, 2),
    "edges": ([[n] for n in (1, 63, 64, 65, 127, 128, 129)], list(range(8)), [[n] for n in (64, 1, 65, 63, 128, 2, 200)], [1] * 7, 2, 1),
    "empty_prefixes": ([[0, 100], [77, 0], [0, 0]], [0, 2, 4, 5], [[3, 9]] * 6, [1] * 6, 4, 2),
    "nothing_at_all": ([[0]], [0, 2], [[0], [3], [0]], [1, 1, 1], 2, 1),
    "some_without": ([[90], [130]], [1, 3, 4], [[20]] * 6, [1, 2, 0, 3, 1, 2], 3, 1),
    "runs_of_none": ([[90], [130], [64], [40]], [0, 0, 3, 3, 5], [[20]] * 5, [1] * 5, 4, 1),
    "more_tokens_than_held": ([[70]], [0, 3], [[1], [0], [2]], [4, 3, 2], 2, 1),
    "rows_17": ([[300]], [0, 17], [[30]] * 17, [1] * 17, 1, 1),
    "rows_64": ([[500, 77]], [0, 16], [[30, 7]] * 16, [1] * 16, 8, 2),
    "rows_100": ([[500, 200]], [0, 25], [[30, 65]] * 25, [1] * 25, 8, 2),
    "rows_128": ([[700]], [0, 32], [[30]] * 32, [1] * 32, 4, 1),
    "rows_129": ([[700], [300]], [0, 129, 131], [[3]] * 131, [1] * 131, 1, 1),
    "rows_400_uneven": ([[700, 1, 333], [64, 900, 128]], [2, 30, 55], [[9, 20, 30]] * 57, [2] * 57, 12, 3),
    "long": ([[6000, 2500]], [0, 70], [[80, 90]] * 70, [1] * 70, 8, 2),
    "long_few": ([[9000, 70]], [0, 3], [[300, 5000]] * 3, [1] * 3, 4, 2),
    "many_heads": ([[100] * 4, [30] * 4], [0, 290, 300], [[5, 70, 1, 20]] * 310, [1] * 310, 4, 4),
    "many_prefixes": ([[70, 5]] * 300, list(range(301)), [[5, 70]] * 300, [1] * 300, 4, 2),
    "many_prefixes_rows": ([[70]] * 40, [20 * x for x in range(41)], [[9]] * 800, [1] * 800, 1, 1),
    "rows_200_short": ([[40, 300], [0, 64]], [0, 25, 50], [[9, 2]] * 50, [1] * 50, 16, 2),
    "draft": ([[400]], [0, 9], [[40]] * 9, [3, 1, 4, 1, 5, 0, 2, 6, 5], 7, 1),
    "pieces_of_prompts": ([[200]], [0, 2], [[64], [150]], [64, 100], 4, 1),
}


@FORMATS
@pytest.mark.parametrize("block", [128, 64])
@pytest.mark.parametrize("name", CASES)
def test_sizes(name, block, fmt):
    plens, groups, lens, new, hq, hkv = CASES[name]
    rng = np.random.default_rng([fmt, block, len(name)])
    prefix, c = filled(rng, plens, block, fmt), filled(rng, lens, block, fmt)
    pre, dev = Device(prefix), Device(c)
    new = np.array(new)
    T = int(new.sum())
    q, q64 = bf16(rng.standard_normal((T, hq, D)))
    step, cu = step_of(dev, new, hq, len(set(new.tolist())) > 1)
    out, lse = call(pre, groups, dev, step, q.to(DEV))
    kv_of = np.arange(hq) * hkv // hq
    want = orc.cache_shared(prefix, groups, c, q64, cu, kv_of)
    check(want, out, lse, slice(0, T), int(np.max(plens) + np.max(lens)), HALF, LIFT)


# By what the tables have room for, more rows are worked on 128 at a time, and prefixes and own tokens in two launches.
ROOMY = {  # ..., pages that tables have room for: of the prefixes, of the own tokens
    "rows_128": ([[250, 70]] * 3, [0, 30, 41, 70], [[9, 70]] * 72, [1] * 72, 8, 2, 4096, 4),
    "rows_128_uneven": ([[1, 0, 333], [64, 900, 128]], [2, 30, 55], [[9, 20, 30]] * 57, [2] * 57, 12, 3, 2000, 4),
    "rows_128_of_many": ([[130]] * 20, [15 * x for x in range(21)], [[20]] * 300, [1] * 300, 4, 1, 4000, 2),
    "rows_128_pieces": ([[200]], [0, 2], [[64], [150]], [64, 100], 4, 1, 4096, 4),
    "rows_16": ([[100, 30]] * 30, [2 * x for x in range(31)], [[30, 200]] * 62, [1] * 62, 8, 2, 600, 100),
    "rows_32": ([[100, 30]] * 10, [7 * x for x in range(11)], [[30, 200]] * 70, [1] * 70, 8, 2, 1500, 5),
    "rows_128_drafts": ([[300, 200], [64, 700]], [1, 9, 20], [[30, 200], [0, 5], [500, 64], [129, 3]] * 6, [5, 6, 7, 2] * 6, 8, 2, 4000, 30),
    "rows_128_drafts_of_many": ([[130]] * 20, [5 * x for x in range(21)], [[20], [90]] * 60, [20] * 120, 4, 1, 4000, 1100),
    "rows_128_drafts_in_little": ([[300, 200]], [0, 40], [[30, 200], [0, 5], [250, 64], [129, 3]] * 11, [6, 5, 7, 0] * 11, 8, 2, 4000, 4),
    "rows_32_own_too": ([[100, 30]] * 5, [2 * x for x in range(6)], [[30, 200]] * 10, [5] * 10, 8, 2, 1500, 1500),
}


@FORMATS
@pytest.mark.parametrize("block", [128, 64])
@pytest.mark.parametrize("name", ROOMY)
def test_tables_with_room(name, block, fmt):
    plens, groups, lens, new, hq, hkv, prefix_pages, own_pages = ROOMY[name]
    rng = np.random.default_rng([fmt, block, len(name)])
    if name == "rows_128_uneven":
        prefix_pages *= 2
    prefix, c = filled(rng, plens, block, fmt, max_pages=prefix_pages, extra_pages=1), filled(rng, lens, block, fmt, max_pages=max(own_pages, 200 // block + 1))
    pre, dev = Device(prefix), Device(c)
    T = int(np.sum(new))
    q, q64 = bf16(rng.standard_normal((T, hq, D)))
    step, cu = step_of(dev, new, hq, len(set(new)) > 1)
    out, lse = call(pre, groups, dev, step, q.to(DEV))
    want = orc.cache_shared(prefix, groups, c, q64, cu, np.arange(hq) * hkv // hq)
    check(want, out, lse, slice(0, T), int(np.max(plens) + np.max(lens)), HALF, LIFT)


@FORMATS
def test_shares_of_many_pages(fmt):
    """A prefix so long that a workgroup's share has more pages than are looked up at once, some of scales that fp16 does not hold; a few
    rows against their products in 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(fmt)
    n, P, hq, hkv, block = 512, 100001, 8, 2, 64
    pages = -(-P // block)
    codes = lambda: (torch.randint(0, 256, (hkv * pages, block, D), device=DEV, generator=gen) % 127
                     + 128 * torch.randint(0, 2, (hkv * pages, block, D), device=DEV, generator=gen)).to(torch.uint8)
    k, v = codes(), codes()
    ks = torch.exp2(torch.randint(-9, -6, (hkv * pages,), device=DEV, generator=gen).float())
    vs = torch.exp2(torch.randint(-9, -6, (hkv * pages,), device=DEV, generator=gen).float())
    table = torch.randperm(hkv * pages, device=DEV, generator=gen).to(torch.int32).view(1, hkv, pages)
    vs[table[0, 1, pages // 2].long()] = 2.0 ** -30
    lens = torch.full((1, hkv), P, dtype=torch.int32, device=DEV)
    prefix = S.Cache(k, v, ks, vs, table, lens, 1, hkv, block, pages, hkv * pages, S.SHPLB_CACHE_E4M3 if fmt == E4M3 else S.SHPLB_CACHE_INT8)
    own = Device(cache_oracle.CacheState(*(np.zeros((1, block, D), np.uint8),) * 2, np.ones(1), np.ones(1), np.full((n, hkv, 1), -1, np.int32), np.zeros((n, hkv), np.int32), fmt))
    q = torch.randn((n, hq, D), device=DEV, generator=gen).to(torch.bfloat16)
    step = S.Step(n, hq, hkv)
    out, lse = torch.zeros_like(q), torch.zeros((hq, n), device=DEV)
    ws = torch.empty(S.shplb_cache_attn_shared_workspace_bytes(prefix, own.cache, step), dtype=torch.uint8, device=DEV)
    S.shplb_cache_attn_shared(prefix, cu_of([0, n]), own.cache, step, q, out, lse, ws, stream())
    value = torch.from_numpy(cache_oracle.decode(np.arange(256), fmt)).to(DEV)
    rows = [0, 1, 77, 128, 300, 511]
    want = orc.Result(np.zeros((len(rows), hq, D)))
    for h in range(hkv):
        at = table[0, h].long()
        kh, vh = ((value[x[at].long()] * sc[at].double()[:, None, None]).view(-1, D)[:P] for x, sc in ((k, ks), (v, vs)))
        for i, r in enumerate(rows):
            for x in range(4 * h, 4 * h + 4):
                want.put(i, x, q[r, x].double().cpu().numpy(), kh.cpu().numpy(), vh.cpu().numpy(), D ** -0.5, True)
    check(want, out[rows].double().cpu().numpy(), lse[:, rows].double().cpu().numpy(), slice(0, len(rows)), P, HALF, LIFT)


def test_blocks_strides_mapped_heads_scale_rows_behind():
    rng = np.random.default_rng(4)
    kv_of = [2, 0, 0, 2, 0]                    # one KV head without query heads
    prefix = filled(rng, [[300, 50, 77]], 64, E4M3)
    c = filled(rng, [[100, 50, 300], [80, 1, 129], [9, 9, 9]], 128, E4M3)
    pre, dev = Device(prefix), Device(c)
    q, q64 = bf16(rng.standard_normal((8, 5, D)))
    qd, wide = strided(q, 4)
    step, cu = step_of(dev, [2, 3, 1], 5, True, behind=2, q_stride_t=wide.shape[1] * D, softmax_scale=0.2, kv_head_of=kv_of)
    out = torch.full_like(wide, 5.0)
    S.shplb_cache_attn_shared(pre.cache, cu_of([0, 2]), dev.cache, step, qd, out[:, 2:7], None, workspace(pre, dev, step), stream())
    want = orc.cache_shared(prefix, [0, 2], c, q64, cu, kv_of, 0.2)
    check(want, out[:, 2:7].double().cpu().numpy(), None, slice(0, 6), 600, HALF, LIFT)
    assert (out[6:] == 5).all() and (out[:, :2] == 5).all() and (out[:, 7:] == 5).all()


@FORMATS
@pytest.mark.parametrize("each", [1, 40])
def test_damage_reaches_those_who_see_it(fmt, each):
    """Lengths that cannot be, pages that are not there or have a scale of NaN, in prefixes and in own tokens."""
    rng = np.random.default_rng(5)
    plens = [[300], [-1], [1000], [300], [300], [300]]
    prefix = filled(rng, np.clip(plens, 0, 384), 64, fmt, max_pages=6)
    prefix.lens[:] = plens
    prefix.table[3, 0, 2] = -1
    prefix.k_scale[prefix.table[4, 0, 0]] = np.nan
    prefix.v_scale[prefix.table[5, 0, 4]] = np.nan
    n = 6 * each + 1
    c = filled(rng, [[70]] * n, 64, fmt)
    c.lens[0, 0] = -5
    c.table[each - 1, 0, 1] = 10 ** 6
    pre, dev = Device(prefix), Device(c)
    q, q64 = bf16(rng.standard_normal((n, 2, D)))
    step, cu = step_of(dev, [1] * n, 2, False)
    groups = [each * x for x in range(7)]
    want = orc.cache_shared(prefix, groups, c, q64, cu, [0, 0])
    assert np.isfinite(want.out[-1]).all() and np.isnan(want.out[each:6 * each]).all()
    check(want, *call(pre, groups, dev, step, q.to(DEV)), slice(0, n), 400, HALF, LIFT)


def test_offsets_out_of_range():
    """cu_prefix outside the sequences is taken as their ends; cu_tokens that go backwards read and write nothing outside."""
    rng = np.random.default_rng(6)
    prefix, c = filled(rng, [[90], [64]], 64, E4M3), filled(rng, [[20]] * 4, 64, E4M3)
    pre, dev = Device(prefix), Device(c)
    q, q64 = bf16(rng.standard_normal((4, 2, D)))
    step, cu = step_of(dev, [1] * 4, 2, False)
    got = call(pre, [-5, 3, 99], dev, step, q.to(DEV))
    check(orc.cache_shared(prefix, [0, 3, 4], c, q64, cu, [0, 0]), *got, slice(0, 4), 110, HALF, LIFT)
    step = S.Step(4, 2, 1, 4, 2, torch.tensor([0, 3, 1, -7, 99], dtype=torch.int32, device=DEV))
    for groups in ([0, 2, 4], [3, 1, 2]):
        for left in (0xff, 0x7f, 0x01):
            call(pre, groups, dev, step, q.to(DEV), workspace(pre, dev, step).fill_(left))


@FORMATS
@pytest.mark.parametrize("new,room", [(1, 4), (6, 4), (6, 40)], ids=["tokens", "drafts_in_little", "drafts"])
def test_damage_where_128_rows_are_taken_together(fmt, new, room):
    rng = np.random.default_rng(16)
    plens = [[300], [-1], [10 ** 6], [300], [300], [300]]
    prefix = filled(rng, np.where(np.array(plens) == 300, 300, 0), 64, fmt, max_pages=4000)
    prefix.lens[:] = plens
    prefix.table[3, 0, 2] = -1
    prefix.k_scale[prefix.table[4, 0, 0]] = np.nan
    prefix.v_scale[prefix.table[5, 0, 4]] = np.nan
    n = 6 * 25 + 1
    c = filled(rng, [[70]] * n, 64, fmt, max_pages=room)
    c.lens[0, 0], c.lens[1, 0] = -5, 64 * room + 1
    c.table[24, 0, 1] = 10 ** 6
    pre, dev = Device(prefix), Device(c)
    q, q64 = bf16(rng.standard_normal((new * n, 4, D)))
    step, cu = step_of(dev, [new] * n, 4, False)
    groups = [25 * x for x in range(7)]
    want = orc.cache_shared(prefix, groups, c, q64, cu, [0] * 4)
    assert np.isfinite(want.out[-1]).all() and np.isfinite(want.out[2 * new]).all() and np.isnan(want.out[25 * new:150 * new]).any(-1).all()
    check(want, *call(pre, groups, dev, step, q.to(DEV)), slice(0, new * n), 400, HALF, LIFT)
    cut = torch.from_numpy(rng.integers(-9, new * n + 9, n + 1).astype(np.int32)).to(DEV)    # offsets in no order: nothing outside is read or written
    step = S.Step(n, 4, 1, new * n, 2 * new, cut)
    for left in (0xff, 0x7f, 0x01):
        call(pre, groups[::-1] if left == 1 else groups, dev, step, q.to(DEV), workspace(pre, dev, step).fill_(left))


@pytest.mark.parametrize("n,room", [(4, 0), (30, 0), (80, 4000)], ids=["rows_8", "rows_60", "rows_160_in_128"])
def test_a_pool_past_32_bits_and_queries_of_nan(n, room):
    rng = np.random.default_rng(22)
    prefix = filled(rng, [[700, 300]], 128, cache_oracle.INT8, max_pages=max(room, 6))
    c = filled(rng, [[9 + 5 * x % 140, 1 + 7 * x % 90] for x in range(n)], 64, cache_oracle.INT8)
    pre, dev = in_a_large_pool(prefix), in_a_large_pool(c)
    q, _ = bf16(rng.standard_normal((n, 4, D)))
    q[2, 1, 77] = np.nan
    step, cu = step_of(dev, [1] * n, 4, False)
    want = orc.cache_shared(prefix, [0, n], c, q.double().numpy(), cu, [0, 0, 1, 1])
    assert np.isnan(want.out[2, 1]).all() and np.isfinite(want.out[2, 0]).all()
    check(want, *call(pre, [0, n], dev, step, q.to(DEV)), slice(0, n), 900, HALF, LIFT)


def test_large_scales_and_queries():
    rng = np.random.default_rng(7)
    for size, qsize, other in ((2.0 ** 40, 2.0 ** -40, 2.0 ** 40), (2.0 ** -60, 2.0 ** 60, 2.0 ** -60), (1.0, 300.0, 1.0), (2.0 ** -100, 1.0, 1.0),
                               (2.0 ** 12, 1e-3, 2.0 ** -12)):
        for n in (3, 50):
            prefix, c = filled(rng, [[500, 1000]], 128, E4M3, size=size), filled(rng, [[100, 30]] * n, 128, E4M3, size=other)
            pre, dev = Device(prefix), Device(c)
            q, q64 = bf16(rng.standard_normal((n, 8, D)) * qsize)
            step, cu = step_of(dev, [1] * n, 8, False)
            want = orc.cache_shared(prefix, [0, n], c, q64, cu, np.arange(8) // 4)
            check(want, *call(pre, [0, n], dev, step, q.to(DEV)), slice(0, n), 1100, HALF, LIFT)


def test_as_one_sequence():
    """A prefix and one sequence behind it give what the cache gives of both in one table."""
    rng = np.random.default_rng(8)
    c = filled(rng, [[900, 900]], 64, E4M3)
    both = Device(c)
    prefix = cache_oracle.CacheState(c.k_pages, c.v_pages, c.k_scale, c.v_scale, c.table[:, :, :10].copy(), np.full((1, 2), 640, np.int32), E4M3)
    own = cache_oracle.CacheState(c.k_pages, c.v_pages, c.k_scale, c.v_scale, c.table[:, :, 10:].copy(), np.full((1, 2), 260, np.int32), E4M3)
    pre, dev = Device(prefix), Device(own)
    q, q64 = bf16(rng.standard_normal((3, 8, D)))
    step, cu = step_of(dev, [3], 8, False)
    got = call(pre, [0, 1], dev, step, q.to(DEV))
    want = orc.cache_shared(prefix, [0, 1], own, q64, cu, np.arange(8) // 4)
    check(want, *got, slice(0, 3), 900, HALF, LIFT)
    out, lse = torch.zeros_like(q, device=DEV), torch.zeros((8, 3), device=DEV)
    ws = torch.empty(S.shplb_cache_attn_workspace_bytes(both.cache, step), dtype=torch.uint8, device=DEV)
    S.shplb_cache_attn(both.cache, step, q.to(DEV), out, lse, None, None, ws, stream())
    check(want, out.double().cpu().numpy(), lse.double().cpu().numpy(), slice(0, 3), 900, HALF, LIFT)


def test_samples_of_a_prompt_token_after_token():
    """As it is used: the prompt is appended once, samples go on from it, append and attention in one captured step."""
    rng = np.random.default_rng(9)
    P, n, hq, hkv, steps = 333, 20, 8, 2, 5
    (pk, pk64), (pv, pv64) = (bf16(rng.standard_normal((P, hkv, D))) for _ in "kv")
    z = lambda m: np.zeros((m, 128, D), np.uint8)
    prefix = cache_oracle.CacheState(z(6), z(6), np.ones(6), np.ones(6), np.arange(6, dtype=np.int32).reshape(1, 2, 3), np.full((1, 2), P, np.int32), E4M3)
    c = cache_oracle.CacheState(z(40), z(40), np.ones(40), np.ones(40), np.arange(40, dtype=np.int32).reshape(20, 2, 1), np.zeros((20, 2), np.int32), E4M3)
    pre, dev = Device(prefix), Device(c)
    S.shplb_cache_append(pre.cache, S.Step(1, hq, hkv, max_tokens=P), pk.to(DEV), pv.to(DEV), stream())
    cache_oracle.append(prefix, pk64, pv64, [0, P])
    pre.check_same(prefix)
    step, cu = step_of(dev, [1] * n, hq, False)
    ws, groups = workspace(pre, dev, step), cu_of([0, n])
    q, k, v = (torch.zeros((n, h, D), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv))
    out, lse = torch.zeros_like(q), torch.zeros((hq, n), device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.shplb_cache_append(dev.cache, step, k, v, stream())
        S.shplb_cache_attn_shared(pre.cache, groups, dev.cache, step, q, out, lse, ws, stream())
    for t in range(steps):
        (a, a64), (b, b64), (x, x64) = (bf16(rng.standard_normal((n, h, D))) for h in (hkv, hkv, hq))
        k.copy_(a); v.copy_(b); q.copy_(x)
        dev.lens += 1
        c.lens += 1
        graph.replay()
        torch.cuda.synchronize()
        cache_oracle.append(c, a64, b64, cu)
        got = out.double().cpu().numpy(), lse.double().cpu().numpy()
        check(orc.cache_shared(prefix, [0, n], c, x64, cu, np.arange(hq) // 4), *got, slice(0, n), P + steps, HALF, LIFT)
        other, again, again_lse, mine = torch.cuda.Stream(), torch.zeros_like(q), torch.zeros_like(lse), workspace(pre, dev, step)
        other.wait_stream(stream())
        S.shplb_cache_attn_shared(pre.cache, groups, dev.cache, step, q, again, again_lse, mine, other)
        torch.cuda.synchronize()
        assert (again == out).all() and (again_lse == lse).all()
    dev.check_same(c)


class Guarded:
    """A buffer with a pattern in front of it and behind it."""
    ROOM = 1 << 16

    def __init__(self, n_bytes, fill):
        self.all = torch.full((2 * self.ROOM + -(-n_bytes // 256) * 256,), 0xa5, dtype=torch.uint8, device=DEV)
        self.end = self.ROOM + n_bytes
        self.bytes = self.all[self.ROOM:self.end]
        self.bytes.fill_(fill)

    def check(self):
        assert (self.all[:self.ROOM] == 0xa5).all() and (self.all[self.end:] == 0xa5).all()


def guarded_call(pre, groups, dev, step, q, left):
    """out, lse (0x41414141 where nothing was written), the workspace's bytes being `left`: nothing around them is written."""
    T, heads = q.shape[0], q.shape[1]
    out, lse, ws = (Guarded(n, f) for n, f in ((T * heads * D * 2, 0x41), (T * heads * 4, 0x41),
                                              (S.shplb_cache_attn_shared_workspace_bytes(pre.cache, dev.cache, step), left)))
    o, l = out.bytes.view(torch.bfloat16).view(T, heads, D), lse.bytes.view(torch.float32).view(heads, T)
    S.shplb_cache_attn_shared(pre.cache, cu_of(groups), dev.cache, step, q, o, l, ws.bytes, stream())
    torch.cuda.synchronize()
    for x in (out, lse, ws):
        x.check()
    return o, l


OVERLAPPING = {  # prefixes, tokens of each, KV heads, sequences, query heads: rows of a prefix's tile as the names say
    "rows_16": (600, 150, 2, 40, 8),
    "rows_32": (20, 200, 2, 50, 16),
    "rows_128": (50, 5120, 1, 700, 4),
}


@FORMATS
@pytest.mark.parametrize("name", OVERLAPPING)
def test_groups_that_overlap(name, fmt):
    """cu_prefix that goes to and fro, so that half of the prefixes have all sequences: many times the work that the call is sized for.  It ends, and
    nothing outside is written; sequences behind the last group are what they are without."""
    n_pre, tokens, hkv, n, hq = OVERLAPPING[name]
    rng = np.random.default_rng(17)
    prefix = filled(rng, [[tokens] * hkv], 64, fmt, spare=0)
    c = filled(rng, [[20] * hkv] * (n + 3), 64, fmt)
    prefix.table, prefix.lens = np.repeat(prefix.table, n_pre, 0), np.repeat(prefix.lens, n_pre, 0)
    pre, dev = Device(prefix), Device(c)
    q, q64 = bf16(rng.standard_normal((n + 3, hq, D)))
    step, cu = step_of(dev, [1] * (n + 3), hq, False)
    groups = [n * (x % 2) for x in range(n_pre + 1)]
    o, l = guarded_call(pre, groups, dev, step, q.to(DEV), 0x7f)
    want = orc.cache_shared(prefix, [0], c, q64, cu, np.arange(hq) * hkv // hq)
    check(want, o.double().cpu().numpy(), l.double().cpu().numpy(), slice(n, n + 3), 84, HALF, LIFT)


def without_order(prefix, groups, c, q64, cut, most_new):
    """What rows get where cu_tokens (cut) and cu_prefix are in no order, as far as it is defined: those of one sequence, of one prefix's rows at most.
    A sequence's rows begin at its offset and are max_tokens at most, a prefix's go from the offset of its first sequence to that of the one
    behind its last; rows of a sequence outside of its prefix's are NaN.  Returns it, and of each row what it is: -1 of no sequence, 1 defined."""
    T, heads = q64.shape[:2]
    inside = lambda x: min(max(int(x), 0), T)
    owners, fronts = ([[] for _ in range(T)] for _ in "of")
    for s in range(len(cut) - 1):
        a = inside(cut[s])
        b = a + min(max(min(int(cut[s + 1]), T) - a, 0), most_new)
        for r in range(a, b):
            owners[r].append((s, r - a, b - a))
    for g in range(len(groups) - 1):
        if groups[g] < groups[g + 1]:
            for r in range(inside(cut[groups[g]]), inside(cut[groups[g + 1]])):
                fronts[r].append(g)
    want, kind = orc.Result(q64), np.zeros(T, int)
    for r in range(T):
        if not owners[r]:
            kind[r] = -1
        if len(owners[r]) != 1 or len(fronts[r]) > 1:
            continue
        kind[r] = 1
        s, j, n = owners[r][0]
        of = [g for g in range(len(groups) - 1) if groups[g] <= s < groups[g + 1]]
        if of and fronts[r] != of:
            want.out[r], want.lse[:, r] = np.nan, np.nan
            continue
        parts = [orc._values_at(prefix, g, 0, np.arange(int(prefix.lens[g, 0]))) for g in of]
        length = int(c.lens[s, 0])
        parts.append([x[:max(0, length - n + 1 + j)] for x in orc._values_at(c, s, 0, np.arange(length))])
        k, v = (np.concatenate([p[x] for p in parts]) for x in (0, 1))
        for h in range(heads):
            want.put(r, h, q64[r, h], k, v, D ** -0.5, True)
    return want, kind


@FORMATS
@pytest.mark.parametrize("n,new,heads,room", [(40, 1, 2, 2), (40, 6, 4, 2), (150, 1, 4, 4), (150, 6, 4, 4), (150, 6, 4, 40)],
                         ids=["rows_16", "rows_32", "rows_128", "rows_128_drafts_in_little", "rows_128_drafts"])
def test_offsets_in_no_order(n, new, heads, room, fmt):
    """cu_tokens in no order, whatever the workspace holds: rows of one sequence and of one prefix at most are right, those of none stay as they were,
    and nothing is written around the buffers."""
    rng = np.random.default_rng([25, n, new])
    large = n > 100
    prefix = filled(rng, [[300], [70], [1]], 64, fmt, max_pages=4000 if large else 5)
    c = filled(rng, rng.integers(0, 120, (n, 1)), 64, fmt, max_pages=room)
    pre, dev = Device(prefix), Device(c)
    T = new * n
    q, q64 = bf16(rng.standard_normal((T, heads, D)))
    groups = [0, n // 3, n // 2, n - 5]
    met = np.zeros(3, int)
    for left in (0xff, 0x7f, 0x01):
        cut = rng.integers(-9, T + 9, n + 1).astype(np.int32)
        ends = np.array([0, n // 3, n // 2, n - 5])
        cut[ends] = np.sort(cut[ends])         # the prefixes' rows are in order
        step = S.Step(n, heads, 1, T, 2 * new, torch.from_numpy(cut).to(DEV))
        want, kind = without_order(prefix, groups, c, q64, cut, 2 * new)
        o, l = guarded_call(pre, groups, dev, step, q.to(DEV), left)
        assert (o[torch.from_numpy(kind < 0).to(DEV)].view(torch.uint8) == 0x41).all()
        rows = np.flatnonzero(kind == 1)
        check(want, o.double().cpu().numpy(), l.double().cpu().numpy(), rows, 420, HALF, LIFT)
        met += [(kind < 0).sum(), np.isnan(want.out[rows, 0, 0]).sum(), np.isfinite(want.out[rows, 0, 0]).sum()]
    assert (met > 0).all()


@FORMATS
@pytest.mark.parametrize("n,room", [(2, 0), (12, 0), (60, 4000)], ids=["rows_8", "rows_48", "rows_240_in_128"])
@pytest.mark.parametrize("size", [(10, 10), (15, 16), (16, 20), (40, 40), (100, -30), (-60, 115)])
def test_scores_that_a_rounding_moves_by_more_than_one(size, n, room, fmt):
    """... those of the prefix the largest for some, of its own tokens for others."""
    rng = np.random.default_rng([28, *(abs(x) for x in size)])
    for order in ("any", "rising", "below_zero"):
        prefix, c = filled(rng, [[700]], 64, fmt, max_pages=max(room, 12)), filled(rng, [[9 + x % 100] for x in range(n)], 64, fmt)
        for x in (prefix, c):
            cu = np.concatenate([[0], np.cumsum(x.lens[:, 0])])
            cache_oracle.append(x, bf16(far_apart(rng, (int(cu[-1]), 1), size[0], order))[1], bf16(rng.standard_normal((int(cu[-1]), 1, D)))[1], cu)
        pre, dev = Device(prefix), Device(c)
        q, q64 = bf16(far_apart(rng, (n, 4), size[1], "any"))
        step, cu = step_of(dev, [1] * n, 4, False)
        want = orc.cache_shared(prefix, [0, n], c, q64, cu, [0] * 4)
        check_far(want, *call(pre, [0, n], dev, step, q.to(DEV)), slice(0, n), HALF)
