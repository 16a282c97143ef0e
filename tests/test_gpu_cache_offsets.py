"""Offsets of a step's sequences that are not what they should be: outside the tensors' rows nothing is read and nothing written."""
import numpy as np
import pytest
import torch

import paper_2603_10353_amd as S
from cache_harness import D, DEV, Device, attn_workspace, bf16, check_attn, filled
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu
ROWS, MOST, GUARD = 6, 3, 40
LEAST, LARGEST = -2 ** 31, 2 ** 31 - 1
# offsets, and what is left of them inside the rows and within the most tokens of a sequence
OFFSETS = {
    "outside": ([-5, 2, 90, 4], [0, 2, 5, 5]),
    "far_outside": ([LEAST, 2, LARGEST, LEAST], [0, 2, 5, 5]),
    "backwards": ([1, 0, LEAST, 0], [0, 0, 0, 0]),
    "behind": ([6, 7, LARGEST, LARGEST], [0, 0, 0, 0]),
    "from_below": ([LEAST, LEAST, -1, 2], [0, 0, 0, 2]),
}


def guarded(rows, fill):
    """A bf16 tensor [ROWS, heads, 128] between rows of something else, and all of them."""
    whole = torch.full((GUARD + rows.shape[0] + GUARD, *rows.shape[1:]), fill, dtype=rows.dtype, device=DEV)
    whole[GUARD:-GUARD] = rows.to(DEV)
    return whole[GUARD:-GUARD], whole


def guards_hold(whole, fill):
    return (whole[:GUARD] == fill).all() and (whole[-GUARD:] == fill).all()


@pytest.mark.parametrize("room", [None, 64])
@pytest.mark.parametrize("hq", [4, 16])                  # 6 and 24 rows of a KV head
@pytest.mark.parametrize("name", OFFSETS)
def test_offsets(name, hq, room):
    print("case", name, hq, room, flush=True)
    rng = np.random.default_rng([len(name), hq])
    offsets, inside = (np.array(x) for x in OFFSETS[name])
    c = filled(rng, [[200, 90], [64, 150], [130, 77]], 64, orc.E4M3, max_pages=room)
    dev = Device(c)
    step = S.Step(3, hq, 2, ROWS, MOST, torch.tensor(offsets, dtype=torch.int32, device=DEV))
    q, q64 = bf16(rng.standard_normal((ROWS, hq, D)))
    qd, _ = guarded(q, float("nan"))
    out, whole = guarded(torch.full((ROWS, hq, D), 9.0, dtype=torch.bfloat16), 9.0)
    lse = torch.full((GUARD + hq * ROWS + GUARD,), 9.0, device=DEV)
    w = rng.random((3, 2, c.capacity)).astype(np.float32)
    w_out = torch.full(w.shape, 9.0, device=DEV)
    stream = torch.cuda.current_stream()
    S.shplb_cache_attn(dev.cache, step, qd, out, lse[GUARD:-GUARD], torch.from_numpy(w).to(DEV), w_out, attn_workspace(dev, step), stream)
    n = int(inside[-1])
    got_lse = lse[GUARD:-GUARD].view(hq, ROWS)
    assert guards_hold(whole, 9) and guards_hold(lse, 9) and (out[n:] == 9).all() and (got_lse[:, n:] == 9).all()
    check_attn(c, out.double().cpu().numpy(), got_lse.double().cpu().numpy(), q64, inside, [h // (hq // 2) for h in range(hq)],
               got_weight=w_out.double().cpu().numpy(), weight_in=w)
    back = [guarded(torch.full((ROWS, 2, D), 9.0, dtype=torch.bfloat16), 9.0) for _ in "kv"]
    S.shplb_cache_load(dev.cache, step, back[0][0], back[1][0], stream)
    want = [np.full((ROWS, 2, D), 9.0) for _ in "kv"]
    orc.load(c, *want, inside)
    for (mine, whole), theirs in zip(back, want):
        np.testing.assert_array_equal(mine.double().cpu().numpy(), theirs)
        assert guards_hold(whole, 9)
    (k, k64), (v, v64) = (bf16(rng.standard_normal((ROWS, 2, D))) for _ in "kv")
    S.shplb_cache_append(dev.cache, step, guarded(k, float("nan"))[0], guarded(v, float("nan"))[0], stream)
    torch.cuda.synchronize()
    orc.append(c, k64, v64, inside)
    dev.check_same(c)
