"""GPU parity of attention over the cache where the scores themselves are the difficulty."""
import numpy as np
import pytest
import torch

import paper_2603_10353_amd as S
from cache_harness import D, DEV, Device, attn_workspace, bf16, check_attn, filled, state, step_of
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu
FORMATS = pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8], ids=["e4m3", "int8"])


@FORMATS
@pytest.mark.parametrize("room", [None, 128], ids=["short", "long"])
@pytest.mark.parametrize("tokens", [1, 4, 5, 30])        # 4, 16, 20 and 120 rows of a KV head
def test_scores_that_grow(tokens, room, fmt):
    # every 64 keys weigh 2^10 times what those before them do, so that what was added up so far is scaled down by that each time; the values in
    # front of a head's last 64 keys are as much larger, so that the scaling shows
    rng = np.random.default_rng([tokens, fmt])
    lens = np.array([[1300, 641], [64, 65], [200, 1000]])
    c = state(rng, lens, 64, fmt, max_pages=room)
    most = int(lens.max())
    direction = rng.choice([-1.0, 1.0], size=(3, 2, D))
    from_end = -(-lens // 64)[:, None, :] - 1 - np.arange(most)[None, :, None] // 64                 # [sequence, place, head]
    q = 2.0 * direction[:, None].repeat(tokens, 1).repeat(4, 2) + 0.1 * rng.standard_normal((3, tokens, 8, D))
    step_up = 10 / (2.0 * D / np.sqrt(D) * np.log2(np.e))
    k = -step_up * from_end[..., None] * direction[:, None] + 0.02 * rng.standard_normal((3, most, 2, D))
    v = rng.standard_normal((3, most, 2, D)) * 2.0 ** (10 * np.clip(from_end, 0, 1))[..., None]
    for s in range(3):                                   # heads of lengths of their own: the tokens of each end where it does
        for h in range(2):
            k[s, :, h], v[s, :, h] = (np.roll(x[s, :, h], most - lens[s, h], 0) for x in (k, v))
    (kt, k64), (vt, v64) = (bf16(x.reshape(-1, 2, D)) for x in (k, v))
    orc.append(c, k64, v64, np.arange(4) * most)
    dev = Device(c)
    q, q64 = bf16(q.reshape(-1, 8, D))
    step, cu = step_of(dev, [tokens] * 3, 8, False)
    out = torch.empty((3 * tokens, 8, D), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((8, 3 * tokens), device=DEV)
    w = torch.zeros((3, 2, c.capacity), device=DEV)
    S.shplb_cache_attn(dev.cache, step, q.to(DEV), out, lse, None, w, attn_workspace(dev, step), torch.cuda.current_stream())
    check_attn(c, out.double().cpu().numpy(), lse.double().cpu().numpy(), q64, cu, [h // 4 for h in range(8)],
               got_weight=w.double().cpu().numpy(), weight_in=np.zeros(w.shape, np.float32))


@pytest.mark.parametrize("room", [None, 64], ids=["short", "long"])
def test_as_many_mapped_heads_as_there_may_be(room):
    # 256 query heads, sixteen of each of the first sixteen KV heads; the last one has none
    rng = np.random.default_rng(31)
    c = filled(rng, [[130] * 16 + [70]], 64, orc.E4M3, max_pages=room)
    dev = Device(c)
    kv_of = [h % 16 for h in range(256)]
    q, q64 = bf16(rng.standard_normal((1, 256, D)))
    step, cu = step_of(dev, [1], 256, False, kv_head_of=kv_of)
    w = rng.random((1, 17, c.capacity)).astype(np.float32)
    out, w_out = torch.empty((1, 256, D), dtype=torch.bfloat16, device=DEV), torch.zeros(w.shape, device=DEV)
    S.shplb_cache_attn(dev.cache, step, q.to(DEV), out, None, torch.from_numpy(w).to(DEV), w_out, attn_workspace(dev, step),
                       torch.cuda.current_stream())
    check_attn(c, out.double().cpu().numpy(), None, q64, cu, kv_of, got_weight=w_out.double().cpu().numpy(), weight_in=w)


@FORMATS
@pytest.mark.parametrize("room", [None, 64], ids=["short", "long"])
@pytest.mark.parametrize("tokens", [1, 6])
def test_large_queries_and_large_keys_apart(tokens, room, fmt):
    # queries and keys of 1e30 and more that have no dim in common, or keys of zeros beside one of 3e38 that the row does not see: scores of 0
    rng = np.random.default_rng([tokens, fmt])
    lens = np.array([[200], [64 + tokens]])
    c = state(rng, lens, 64, fmt, max_pages=room)
    k = rng.standard_normal((200 + 64 + tokens, 1, D)) * 1e30
    k[:, :, 64:] = 0.0
    k[200:] = 0.0
    k[-1] = 3e38
    (k, k64), (v, v64) = (bf16(x) for x in (k, rng.standard_normal(k.shape)))
    orc.append(c, k64, v64, np.array([0, 200, 264 + tokens]))
    dev = Device(c)
    q = rng.standard_normal((2 * tokens, 4, D)) * 1e30
    q[:, :, :64] = 0.0
    if tokens == 1:                                      # ... but the last row sees it: not finite, or not at all large
        q[1] = rng.standard_normal((4, D)) * 1e-38
    q, q64 = bf16(q)
    step, cu = step_of(dev, [tokens] * 2, 4, False)
    out = torch.empty((2 * tokens, 4, D), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((4, 2 * tokens), device=DEV)
    w = torch.zeros((2, 1, c.capacity), device=DEV)
    S.shplb_cache_attn(dev.cache, step, q.to(DEV), out, lse, None, w, attn_workspace(dev, step), torch.cuda.current_stream())
    got, got_lse, got_w = (x.double().cpu().numpy() for x in (out, lse, w))
    finite = slice(0, 2 * tokens - (tokens > 1))
    assert np.isfinite(got[finite]).all() and np.isfinite(got_lse[:, finite]).all() and np.isfinite(got_w[0]).all()
    # the first sequence's scores are 0, and so are the second's but for its last row's: means of the values, within bf16's half step and fp16's of
    # equal probabilities
    one = orc.CacheState(c.k_pages, c.v_pages, c.k_scale, c.v_scale, c.table[:1], c.lens[:1], fmt)
    check_attn(one, got[:tokens], got_lse[:, :tokens], q64[:tokens], cu[:2], [0] * 4, got_weight=got_w[:1], weight_in=np.zeros((1, 1, c.capacity)))
    for j in range(tokens - 1):
        values = c.values("v", 1, 0, 65 + j)
        tol = 2.0 ** -8 * np.abs(values.mean(0)) + 2.0 ** -11 * 1.01 * np.abs(values).mean(0)
        assert (np.abs(got[tokens + j] - values.mean(0)) <= tol).all()


@FORMATS
@pytest.mark.parametrize("room", [None, 64], ids=["short", "long"])
@pytest.mark.parametrize("tokens", [1, 6])
@pytest.mark.parametrize("size", [1e-40, 1e-38, 1e-36, 1e-31])
def test_small_queries_and_large_keys(size, tokens, room, fmt):
    # queries down to bf16's subnormals, and keys as large as makes scores of ordinary size of them
    rng = np.random.default_rng([tokens, fmt])
    lens = np.array([[200, 70]])
    c = state(rng, lens, 64, fmt, max_pages=room)
    k = np.clip(rng.standard_normal((200, 2, D)) * min(1 / size, 1e38), -3e38, 3e38)
    (k, k64), (v, v64) = (bf16(x) for x in (k, rng.standard_normal(k.shape)))
    orc.append(c, k64, v64, np.array([0, 200]))
    dev = Device(c)
    q, q64 = bf16(rng.standard_normal((tokens, 8, D)) * size)
    step, cu = step_of(dev, [tokens], 8, False)
    out, lse = torch.empty((tokens, 8, D), dtype=torch.bfloat16, device=DEV), torch.empty((8, tokens), device=DEV)
    w = torch.zeros((1, 2, c.capacity), device=DEV)
    S.shplb_cache_attn(dev.cache, step, q.to(DEV), out, lse, None, w, attn_workspace(dev, step), torch.cuda.current_stream())
    check_attn(c, out.double().cpu().numpy(), lse.double().cpu().numpy(), q64, cu, [h // 4 for h in range(8)],
               got_weight=w.double().cpu().numpy(), weight_in=np.zeros(w.shape, np.float32))


@FORMATS
@pytest.mark.parametrize("room", [None, 128], ids=["short", "long"])
@pytest.mark.parametrize("tokens", [1, 6])
@pytest.mark.parametrize("size", [1e7, 3e8, 1e10, 1e25])
def test_scores_past_24_bits(size, tokens, room, fmt):
    # scores whose last place in fp32 is a factor of two and more between probabilities: nearly all of a row's lies on one key, which may be one of
    # those within that; what comes out is finite
    rng = np.random.default_rng([tokens, fmt])
    lens = np.array([[500, 130], [64, 1000]])
    c = state(rng, lens, 64, fmt, max_pages=room)
    near = np.round(2 * rng.standard_normal((2000, 2, 1))) * 1e-7            # many keys that are nearly the largest
    k = np.sqrt(size) * (1 + near) * rng.choice([-1.0, 1.0], size=(1, 1, D)) * np.ones((1, 1, D))
    k = np.where(rng.random((2000, 2, 1)) < 0.5, k, k * rng.uniform(-1, 1, size=(2000, 2, 1)))
    (k, k64), (v, v64) = (bf16(x) for x in (k, rng.standard_normal(k.shape)))
    orc.append(c, k64, v64, np.array([0, 1000, 2000]))
    dev = Device(c)
    q, q64 = bf16(np.sqrt(size) * rng.standard_normal((2 * tokens, 8, D)))
    step, cu = step_of(dev, [tokens] * 2, 8, False)
    out, lse = torch.empty((2 * tokens, 8, D), dtype=torch.bfloat16, device=DEV), torch.empty((8, 2 * tokens), device=DEV)
    w = rng.uniform(0.5, 1.0, size=(2, 2, c.capacity)).astype(np.float32)
    w_out = torch.zeros(w.shape, device=DEV)
    S.shplb_cache_attn(dev.cache, step, q.to(DEV), out, lse, torch.from_numpy(w).to(DEV), w_out, attn_workspace(dev, step),
                       torch.cuda.current_stream())
    got, got_lse, got_w = (x.double().cpu().numpy() for x in (out, lse, w_out))
    check_attn(c, got, got_lse, q64, cu, [h // 4 for h in range(8)], got_weight=got_w, weight_in=w)
    # every row's weights are those of one softmax
    given = [(got_w[s, h, :lens[s, h]] - w[s, h, :lens[s, h]]).sum() for s in range(2) for h in range(2)]
    assert np.isfinite(got).all() and np.isfinite(got_lse).all() and (np.abs(np.array(given) / (4 * tokens) - 1) < 0.01).all()
