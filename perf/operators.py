"""What is timed of the 8-bit key/value cache: writing tokens into it, reading them back, attention of the next
tokens over it, and eviction by accumulated attention weight.

The cache is a pool of pages.  A page holds `block` tokens of one KV head of one sequence, a byte a value, with one
scale for its keys and one for its values; page_table[s][h][i] is the page of tokens i * block and on, lens[s][h]
the tokens held (those of the present step included).  A scale is the smallest power of two (2^-126 at least) with
which the page's largest value fits the format, so a code is one rounding (to nearest, ties to even) of its value.
Pages that gain tokens keep their scale or take a larger one, with which the older codes are rounded again.

Shapes are those of the benchmark configurations (workloads/synth.py), the head counts of the parity tests, and
generic serving sizes.  The pools' unused bytes hold whatever was there, as they do in a running program.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
D = 128
LARGEST = {"e4m3": 448.0, "int8": 127.0}
SINK = RECENT = 128            # tokens that eviction always keeps: the first and the last ones


def _log_lengths(n, lo, hi, seed):
    r = np.random.Generator(np.random.Philox(key=[seed, 1]))
    return ",".join(str(int(x)) for x in np.exp(r.uniform(math.log(lo), math.log(hi), size=n)))


def listed():
    def case(name, op, lens, new, hq, hkv, block, fmt, **more):
        c = dict(name=name, op=op, lens=lens, new=new, q_heads=hq, kv_heads=hkv, block=block, format=fmt,
                 uneven=False, weights=False, packed=False, keep="", plan_seed=1)
        c.update(more)
        return c

    return [
        # the next token of one short conversation: nothing but latency
        case("attn_one_777", "attn", "777", "1", 32, 8, 128, "e4m3"),
        # plain multi-head attention behind a 2K prompt, fine pages, the other format
        case("attn_mha_2k_b64", "attn", "2048", "1", 8, 8, 64, "int8"),
        # a serving step of many short requests that also keeps the books for a later eviction
        case("attn_batch_48_weights", "attn", _log_lengths(48, 20, 2000, 48), "1", 28, 4, 128, "e4m3", weights=True, packed=True),
        # a large serving batch whose heads were evicted to lengths of their own
        case("attn_batch_128_uneven", "attn", _log_lengths(128, 1000, 16000, 128), "1", 32, 8, 128, "e4m3", uneven=True),
        # the next token of one 128K context
        case("attn_one_128k", "attn", "131072", "1", 32, 8, 128, "e4m3"),
        # the last 32 tokens of a 32K prompt looking back over it, to weigh its tokens before an eviction
        case("attn_window_32k_weights", "attn", "32768", "32", 32, 8, 128, "int8", weights=True),
        # one new token of each of 64 conversations is written, in pages that hold others
        case("append_step_64", "append", _log_lengths(64, 200, 8000, 64), "1", 32, 8, 128, "e4m3", packed=True),
        # a 32K prompt is written as a fused projection leaves it
        case("append_prompt_32k", "append", "32768", "32768", 32, 8, 128, "e4m3", packed=True),
        # a batch of short requests is read back in 16 bits, to be moved or worked on
        case("load_batch_48_b64", "load", _log_lengths(48, 20, 2000, 48), "all", 28, 4, 64, "e4m3"),
        # one long cache is read back
        case("load_64k", "load", "65536", "all", 8, 2, 128, "int8"),
        # a batch of short requests is evicted to a budget per head
        case("evict_batch_48", "evict", _log_lengths(48, 20, 2000, 48), "0", 28, 4, 64, "int8", keep="log:0.2:1"),
        # a 128K context is evicted to the budgets of the headline layer, one head keeping everything
        case("evict_128k", "evict", "131072", "0", 32, 8, 128, "e4m3", keep="log:0.01:0.3:1"),
    ]


def draw(rng):
    """One more case of the same ranges."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["attn", "attn", "attn", "append", "load", "evict"])
    hq, hkv = rng.choice([(32, 8), (28, 4), (40, 8), (8, 8), (8, 2), (16, 4)])
    n = rng.choice([1, 1, 1, 2, 3, 5, 8, 16, 48, 100])
    most = max(64, min(131072, 600000 // (n * hkv)))
    lens = [log(1 if n > 1 else 40, most) for _ in range(n)]
    c = dict(op=op, q_heads=hq, kv_heads=hkv, block=rng.choice([128, 128, 64]), format=rng.choice(["e4m3", "e4m3", "int8"]),
             uneven=rng.random() < 0.3, weights=False, packed=rng.random() < 0.4, keep="", plan_seed=rng.randrange(1 << 20))
    if op == "attn":
        new = rng.choice([1, 1, 1, 1, 2, 3, 4, 7, 8, 16, 32])
        c["new"] = ",".join([str(new)] + [str(rng.randint(0, new)) for _ in lens[1:]]) if rng.random() < 0.3 else str(new)
        c["weights"] = rng.random() < 0.4
    elif op == "append":
        # a step, a piece of a prompt behind what is there, or a whole prompt
        how = rng.choice(["step", "piece", "prompt"])
        lens = [min(x, 32768) for x in lens]
        c["uneven"] = c["uneven"] and how == "step"
        c["new"] = "1" if how == "step" else "all" if how == "prompt" else ",".join(str(rng.randint(i == 0, x)) for i, x in enumerate(lens))
    elif op == "load":
        c["new"] = "all"
    else:
        c["new"] = "0"
        c["keep"] = rng.choice(["log:0.01:0.3", "log:0.02:0.5", "log:0.2:1", "log:0.01:0.3:1", "log:0.05:0.5:1"])
    c["lens"] = ",".join(str(x) for x in lens)
    return c


# ---- what a case's text stands for --------------------------------------------------------------------------------------


def _lens(case):
    return np.array([int(x) for x in case["lens"].split(",")], np.int64)


def _new(case):
    """Tokens of the step, per sequence."""
    lens = _lens(case)
    if case["new"] == "all":
        return lens
    new = np.array([int(x) for x in case["new"].split(",")], np.int64)
    return new if new.size == lens.size else np.full(lens.size, new[0])


def _head_lens(case):
    """Tokens held, per sequence and KV head."""
    lens = np.repeat(_lens(case)[:, None], case["kv_heads"], 1)
    if case["uneven"]:
        f = np.random.Generator(np.random.Philox(key=[case["plan_seed"], 3])).uniform(math.log(0.1), 0.0, size=lens.shape)
        lens = np.maximum(1, (lens * np.exp(f)).astype(np.int64))
    return lens


def _keep(case):
    """Tokens that eviction is to keep, per sequence and KV head."""
    lens = _head_lens(case)
    _, lo, hi, *whole = case["keep"].split(":")
    rng = np.random.Generator(np.random.Philox(key=[case["plan_seed"], 4]))
    f = np.exp(rng.uniform(math.log(float(lo)), math.log(float(hi)), size=lens.shape))
    if whole:
        f[:, rng.choice(lens.shape[1], size=int(whole[0]), replace=False)] = 1.0
    return np.maximum(1, (lens * f).astype(np.int64))


def _kept(case):
    return np.minimum(_head_lens(case), np.maximum(_keep(case), SINK + RECENT))


def _read_back(case):
    """Tokens whose values are read back to see what an operator did, per sequence."""
    if case["op"] == "append":                   # the pages written to, whole
        return np.minimum(_lens(case), _new(case) + case["block"])
    if case["op"] == "evict":
        return _kept(case).max(1)
    return _new(case)


def _cu(n):
    return np.concatenate([[0], np.cumsum(n)])


# ---- the format, as torch has it ----------------------------------------------------------------------------------------


def _power_of_two(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale(amax, fmt):
    """The smallest power of two with which amax fits: amax = m * 2^e with 1/2 <= m < 1, 448 = 7/8 * 2^9, 127 = 127/128 * 2^7."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875) if fmt == "e4m3" else e - 7 + (m > 0.9921875)
    return _power_of_two(torch.where(amax > 0, e.clamp(min=-126), torch.full_like(e, -126)))


def _codes(x, scale, fmt):
    y = x / scale
    return (y.to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().clamp(-127, 127).to(torch.int8)).view(torch.uint8)


def _values(codes, fmt):
    return codes.view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).to(torch.float32)


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _pages(case, head_lens, seed, spare=1):
    """A page table over a pool in no order, and how many pages the pool has.  Entries that no token needs are -1."""
    nb = -(-head_lens // case["block"])
    width = int(nb.max()) + spare
    need = np.arange(width) < nb[..., None] + spare
    table = np.full(need.shape, -1, np.int32)
    n = int(need.sum())
    table[need] = np.random.default_rng([seed, 5]).permutation(n)
    return torch.from_numpy(table).to(DEV), n


def _filled(case, n_pages, table, held, gen, direction, keys):
    """Pages of a running program: tokens of noise, for keys with some that a head's queries look for (the first one
    among them), for values with a small first one; behind the tokens held, whatever bytes there were."""
    block, fmt = case["block"], case["format"]
    pages = torch.randint(0, 256, (n_pages, block, D), device=DEV, generator=gen, dtype=torch.uint8)
    scale = torch.ones(n_pages, device=DEV)
    s, h, i = torch.nonzero(table >= 0, as_tuple=True)
    page, left = table[s, h, i].long(), held[s, h] - i * block
    for at in range(0, page.numel(), 8192):
        part = slice(at, min(at + 8192, page.numel()))
        x = torch.randn((part.stop - at, block, D), device=DEV, generator=gen)
        first = (i[part] == 0)[:, None] & (torch.arange(block, device=DEV) == 0)
        if keys:
            pull = torch.rand((part.stop - at, block), device=DEV, generator=gen)
            pull = torch.where(pull < 0.01, pull * 400, torch.zeros_like(pull))
            x += torch.where(first, 3.0, pull)[..., None] * direction[h[part]][:, None]
        else:
            x = torch.where(first[..., None], x * 0.02, x)
        x = x.to(torch.bfloat16).to(torch.float32)
        there = torch.arange(block, device=DEV) < left[part, None]
        sc = _scale((x.abs() * there[..., None]).amax((1, 2)), fmt)
        pages[page[part]] = torch.where(there[..., None], _codes(x, sc[:, None, None], fmt), pages[page[part]])
        scale[page[part]] = sc
    return pages, scale


def prepare(case, seed):
    hq, hkv, block, fmt, op = (case[x] for x in ("q_heads", "kv_heads", "block", "format", "op"))
    gen = torch.Generator(device=DEV).manual_seed(seed)
    head_lens, new, lens = _head_lens(case), _new(case), _lens(case)
    table, n_pages = _pages(case, head_lens, seed)
    direction = torch.randn((hkv, D), device=DEV, generator=gen)
    direction = 4.0 * direction / direction.norm(dim=1, keepdim=True)
    dev_lens = torch.from_numpy(head_lens.astype(np.int32)).to(DEV)
    held = (dev_lens - torch.from_numpy(new).to(DEV)[:, None]).clamp(min=0) if op == "append" else dev_lens
    k_pages, k_scale = _filled(case, n_pages, table, held, gen, direction, True)
    v_pages, v_scale = _filled(case, n_pages, table, held, gen, direction, False)
    st = dict(case=case, k_pages=k_pages, v_pages=v_pages, k_scale=k_scale, v_scale=v_scale, table=table, lens=dev_lens,
              n_pages=n_pages, total=int(new.sum()), most=int(new.max()), cu_host=_cu(new),
              cu=torch.from_numpy(_cu(new).astype(np.int32)).to(DEV))
    back = _read_back(case)
    if op != "attn":
        st.update(back_total=int(back.sum()), back_most=int(back.max()), back_cu=torch.from_numpy(_cu(back).astype(np.int32)).to(DEV),
                  k_back=torch.zeros((int(back.sum()), hkv, D), dtype=torch.bfloat16, device=DEV))
        st["v_back"] = torch.zeros_like(st["k_back"])
    cap = table.shape[2] * block
    here = torch.arange(cap, device=DEV) < dev_lens[..., None]
    if op == "append":
        qkv = torch.randn((st["total"], (hq if case["packed"] else 0) + 2 * hkv, D), device=DEV, generator=gen)
        qkv *= torch.where(torch.rand((st["total"], 1, 1), device=DEV, generator=gen) < 0.1, 3.0, 1.0)
        st["qkv"] = qkv.to(torch.bfloat16)
        st["k"], st["v"] = st["qkv"][:, -2 * hkv:-hkv], st["qkv"][:, -hkv:]
    elif op == "attn":
        width = hq + 2 * hkv if case["packed"] else hq
        q = torch.randn((st["total"], width, D), device=DEV, generator=gen)
        q[:, :hq] += 0.5 * direction.repeat_interleave(hq // hkv, 0)
        st["qkv"] = q.to(torch.bfloat16)
        st["q"] = st["qkv"][:, :hq]
        st["out"] = torch.zeros_like(st["qkv"])[:, :hq]
        st["lse"] = torch.zeros((hq, st["total"]), device=DEV)
        if case["weights"]:
            st["weight"] = torch.rand(here.shape, device=DEV, generator=gen) * here
            st["weight_out"] = torch.zeros_like(st["weight"])
    elif op == "evict":
        # few tokens hold most of the weight, and some were never looked at
        w = torch.exp(2.0 * torch.randn(here.shape, device=DEV, generator=gen) - 6.0)
        w = torch.where(torch.rand(here.shape, device=DEV, generator=gen) < 0.1, torch.zeros_like(w), w)
        kept = _kept(case)
        to_table, to_pages = _pages(case, kept, seed + 1, spare=0)
        st.update(weight=w, keep=torch.from_numpy(_keep(case).astype(np.int32)).to(DEV), to_table=to_table, to_n_pages=to_pages,
                  to_k_pages=torch.randint(0, 256, (to_pages, block, D), device=DEV, generator=gen, dtype=torch.uint8),
                  to_v_pages=torch.randint(0, 256, (to_pages, block, D), device=DEV, generator=gen, dtype=torch.uint8),
                  to_k_scale=torch.ones(to_pages, device=DEV), to_v_scale=torch.ones(to_pages, device=DEV),
                  to_lens=torch.zeros_like(dev_lens),
                  to_weight=torch.zeros((*to_table.shape[:2], to_table.shape[2] * block), device=DEV),
                  kept=torch.zeros((*to_table.shape[:2], to_table.shape[2] * block), dtype=torch.int32, device=DEV))
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------------


def run(st):
    op = st["case"]["op"]
    if own:
        return _own(st)
    if op == "append":
        _plain_append(st, st["k"], st["k_pages"], st["k_scale"])
        _plain_append(st, st["v"], st["v_pages"], st["v_scale"])
    if op == "attn":
        return _plain_attn(st)
    if op == "evict":
        return _plain_evict(st)
    _plain_load(st, st["k_pages"], st["k_scale"], st["table"], st["lens"], st["k_back"])
    _plain_load(st, st["v_pages"], st["v_scale"], st["table"], st["lens"], st["v_back"])
    return dict(k=st["k_back"], v=st["v_back"])


def _handles(st):
    """What a program makes once and keeps: the cache, the step, a workspace."""
    import paper_2603_10353_amd as S
    case = st["case"]
    hq, hkv, block = case["q_heads"], case["kv_heads"], case["block"]
    fmt = S.SHPLB_CACHE_E4M3 if case["format"] == "e4m3" else S.SHPLB_CACHE_INT8
    n = st["lens"].shape[0]
    even = len(set(np.diff(st["cu_host"]).tolist())) == 1
    st["cache"] = S.Cache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], st["table"], st["lens"], n, hkv,
                          block, st["table"].shape[2], st["n_pages"], fmt)
    if case["op"] != "evict":
        strides = {}
        if "qkv" in st:
            strides = {"q_stride_t" if case["op"] == "attn" else "kv_stride_t": st["qkv"].stride(0)}
        st["step"] = S.Step(n, hq, hkv, st["total"], st["most"], None if even else st["cu"], **strides)
    if case["op"] == "attn":
        st["ws"] = torch.empty(S.shplb_cache_attn_workspace_bytes(st["cache"], st["step"]), dtype=torch.uint8, device=DEV)
    else:
        st["back"] = S.Step(n, hq, hkv, st["back_total"], st["back_most"], st["back_cu"])
    if case["op"] == "evict":
        st["to"] = S.Cache(st["to_k_pages"], st["to_v_pages"], st["to_k_scale"], st["to_v_scale"], st["to_table"],
                           st["to_lens"], n, hkv, block, st["to_table"].shape[2], st["to_n_pages"], fmt)
        st["ws"] = torch.empty(S.shplb_cache_evict_workspace_bytes(st["cache"]), dtype=torch.uint8, device=DEV)
    st["S"] = S


def _own(st):
    if "S" not in st:
        _handles(st)
    S, op, stream = st["S"], st["case"]["op"], torch.cuda.current_stream()
    if op == "attn":
        weights = (st["weight"], st["weight_out"]) if "weight" in st else (None, None)
        S.shplb_cache_attn(st["cache"], st["step"], st["q"], st["out"], st["lse"], *weights, st["ws"], stream)
        return _attn_outputs(st)
    if op == "evict":
        S.shplb_cache_evict(st["cache"], st["weight"], st["keep"], SINK, RECENT, st["to"], st["to_weight"], st["kept"], st["ws"], stream)
        S.shplb_cache_load(st["to"], st["back"], st["k_back"], st["v_back"], stream)
        return _evict_outputs(st)
    if op == "append":
        S.shplb_cache_append(st["cache"], st["step"], st["k"], st["v"], stream)
    S.shplb_cache_load(st["cache"], st["back"], st["k_back"], st["v_back"], stream)
    return dict(k=st["k_back"], v=st["v_back"])


def _attn_outputs(st):
    got = dict(out=st["out"], lse=st["lse"])
    if "weight" in st:
        got["weight"] = st["weight_out"]
    return got


def _evict_outputs(st):
    return dict(k=st["k_back"], v=st["v_back"], lens=st["to_lens"], weight=st["to_weight"], kept=st["kept"])


def _page_values(st, x, scale, which):
    """Values and codes of the pages `which` (any shape; -1 gives page 0)."""
    at = which.clamp(min=0).long()
    return _values(x[at], st["case"]["format"]) * scale[at][..., None, None]


def _plain_append(st, x, pages, scale):
    block, fmt, table = st["case"]["block"], st["case"]["format"], st["table"]
    new = (st["cu"][1:] - st["cu"][:-1])[:, None, None]
    length = st["lens"][..., None]
    start = length - new
    # the pages that the step touches, then their slots
    i = start.clamp(min=0) // block + torch.arange((st["most"] + block - 2) // block + 1, device=DEV)
    touched = (i * block < length) & (new > 0)
    which = table.gather(2, i.clamp(max=table.shape[2] - 1).long())
    pos = i[..., None] * block + torch.arange(block, device=DEV)
    fresh = (pos >= start[..., None]) & (pos < length[..., None]) & touched[..., None]
    old = pos < start[..., None]
    row = (st["cu"][:-1, None, None, None] + pos - start[..., None]).clamp(0, max(st["total"] - 1, 0)).long()
    head = torch.arange(table.shape[1], device=DEV)[None, :, None, None]
    value = torch.where(fresh[..., None], x[row, head].to(torch.float32), 0.0)
    at = which.clamp(min=0).long()
    before = _page_values(st, pages, scale, which)
    sc = _scale(value.abs().amax((3, 4)), fmt)
    sc = torch.where(old[..., 0], torch.maximum(sc, scale[at]), sc)
    value = torch.where(old[..., None], before, value)
    code = torch.where((fresh | old)[..., None], _codes(value, sc[..., None, None], fmt), pages[at])
    pages[which[touched].long()] = code[touched]
    scale[which[touched].long()] = sc[touched]


def _plain_load(st, pages, scale, table, lens, out):
    block, hkv = st["case"]["block"], st["case"]["kv_heads"]
    cu = st["back_cu"].long()
    row = torch.arange(st["back_total"], device=DEV)
    s = torch.searchsorted(cu, row, right=True) - 1
    pos = (row - cu[s + 1])[:, None] + lens[s].long()                          # [rows, heads]
    there = pos >= 0
    pos = pos.clamp(min=0)
    head = torch.arange(hkv, device=DEV)
    page = table[s[:, None], head, pos // block].clamp(min=0).long()
    value = _values(pages[page, pos % block], st["case"]["format"]) * scale[page][..., None]
    out.copy_(torch.where(there[..., None], value.to(torch.bfloat16), out))


def _plain_attn(st):
    case = st["case"]
    block, hq, hkv = case["block"], case["q_heads"], case["kv_heads"]
    table, lens, most = st["table"], st["lens"], st["most"]
    n, cap, group = table.shape[0], table.shape[2] * block, hq // hkv
    pos = torch.arange(cap, device=DEV)
    there = pos < lens[..., None]
    k = _page_values(st, st["k_pages"], st["k_scale"], table).view(n, hkv, cap, D)
    v = _page_values(st, st["v_pages"], st["v_scale"], table).view(n, hkv, cap, D)
    k.masked_fill_(~there[..., None], 0.0)
    v.masked_fill_(~there[..., None], 0.0)
    # queries, padded to the longest run: [sequence, KV head, query, head of the group]
    new = st["cu"][1:] - st["cu"][:-1]
    j = torch.arange(most, device=DEV)
    row = (st["cu"][:-1, None] + j).clamp(max=max(st["total"] - 1, 0)).long()
    q = st["q"][row].to(torch.float32).view(n, most, hkv, group, D).transpose(1, 2).reshape(n, hkv, most * group, D)
    z = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    seen = lens[:, :, None] - new[:, None, None] + 1 + j                       # [n, hkv, most]
    seen = torch.where(j < new[:, None, None], seen, 0).repeat_interleave(group, 2)
    z.masked_fill_(pos >= seen[..., None], -math.inf)
    top = z.amax(3, keepdim=True).clamp(min=-3.0e38)
    p = torch.exp(z - top)
    total = p.sum(3, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    out = torch.matmul(p, v).view(n, hkv, most, group, D).transpose(1, 2).reshape(n, most, hq, D)
    lse = (top + torch.log(total)).view(n, hkv, most, group).transpose(1, 2).reshape(n, most, hq)
    mine = j < new[:, None]
    st["out"][row[mine]] = out[mine].to(torch.bfloat16)
    st["lse"][:, row[mine]] = lse[mine].T
    if "weight" in st:
        st["weight_out"].copy_(torch.where(there, st["weight"] + p.sum(2), st["weight_out"]))
    return _attn_outputs(st)


def _plain_evict(st):
    case = st["case"]
    block, fmt = case["block"], case["format"]
    lens, cap, to_cap = st["lens"], st["weight"].shape[2], st["kept"].shape[2]
    pos = torch.arange(cap, device=DEV)
    n = torch.minimum(lens, st["keep"].clamp(min=SINK + RECENT)).clamp(max=to_cap)
    always = (pos < SINK) | (pos >= lens[..., None] - RECENT)
    w = torch.where(always, math.inf, st["weight"])
    w = torch.where(pos < lens[..., None], w, -math.inf)
    order = torch.sort(w, dim=2, descending=True, stable=True).indices         # ties: the lower position first
    stays = torch.zeros(w.shape, dtype=torch.bool, device=DEV)
    stays.scatter_(2, order, pos < n[..., None])
    s, h, at = torch.nonzero(stays, as_tuple=True)
    to = (torch.cumsum(stays, 2) - 1)[s, h, at]
    st["kept"][s, h, to] = at.to(torch.int32)
    st["to_weight"][s, h, to] = st["weight"][s, h, at]
    st["to_lens"].copy_(n)
    _plain_gather(st, st["k_pages"], st["k_scale"], st["to_k_pages"], st["to_k_scale"], n)
    _plain_gather(st, st["v_pages"], st["v_scale"], st["to_v_pages"], st["to_v_scale"], n)
    _plain_load(st, st["to_k_pages"], st["to_k_scale"], st["to_table"], st["to_lens"], st["k_back"])
    _plain_load(st, st["to_v_pages"], st["to_v_scale"], st["to_table"], st["to_lens"], st["v_back"])
    return _evict_outputs(st)


def _plain_gather(st, pages, scale, to_pages, to_scale, n):
    block, fmt = st["case"]["block"], st["case"]["format"]
    s, h, i = torch.nonzero(st["to_table"] >= 0, as_tuple=True)
    slot = torch.arange(block, device=DEV)
    at = st["kept"].view(*st["kept"].shape[:2], -1, block)[s, h, i].long()     # [pages, block]
    page = st["table"][s[:, None], h[:, None], at // block].clamp(min=0).long()
    there = i[:, None] * block + slot < n[s, h][:, None]
    value = _values(pages[page, at % block], fmt) * scale[page][..., None]
    value = torch.where(there[..., None], value, 0.0)
    sc = _scale(value.abs().amax((1, 2)), fmt)
    which = st["to_table"][s, h, i].long()
    to_pages[which] = torch.where(there[..., None], _codes(value, sc[:, None, None], fmt), to_pages[which])
    to_scale[which] = sc


# ---- cost ---------------------------------------------------------------------------------------------------------------


def work(case):
    """Each byte that an operator needs read once, each one that it makes written once; products of the visible pairs."""
    hq, hkv = case["q_heads"], case["kv_heads"]
    lens, new, op = _head_lens(case), _new(case), case["op"]
    held = int(lens.sum())
    nbytes = flops = 0
    if op == "attn":
        first = lens - new[:, None] + 1                                        # what the first query of a run sees
        low = np.maximum(first, 1)
        pairs = np.where(lens >= low, (low + lens) * (lens - low + 1) // 2, 0)
        pairs = int(np.where(new[:, None] > 0, pairs, 0).sum()) * (hq // hkv)
        nbytes = 2 * D * int(lens[new > 0].sum()) + 2 * 2 * D * hq * int(new.sum()) + (8 * held if case["weights"] else 0)
        flops = 4 * D * pairs
    else:
        back = int(np.minimum(_read_back(case)[:, None], lens if op != "evict" else _kept(case)).sum())
        nbytes = 6 * D * back                                                  # read in 8 bits, written in 16
        if op == "append":
            nbytes += 6 * D * int(np.minimum(new[:, None], lens).sum())
        if op == "evict":
            nbytes += 4 * held + (4 * D + 8) * int(_kept(case).sum())
    return {"bytes": nbytes, "flops": flops}


# ---- the definition in 64 bits, one sequence and head after the other ---------------------------------------------------


def _decoded(codes, fmt):
    """Codes as the numbers they stand for: sign, exponent and three bits below it, or a whole number."""
    c = codes.to(torch.int64)
    if fmt == "int8":
        return torch.where(c > 127, c - 256, c).double()
    e, m = (c >> 3) & 15, (c & 7).double()
    mag = torch.where(e > 0, (1 + m / 8) * torch.exp2((e - 7).double()), m / 512)
    mag = torch.where((c & 127) == 127, math.nan, mag)
    return torch.where(c > 127, -mag, mag)


def _smallest(amax, fmt):
    """The scale, as a float: the least power of two that amax / LARGEST does not pass."""
    return 2.0 ** max(-126, math.ceil(math.log2(amax / LARGEST[fmt]))) if amax > 0 else 2.0 ** -126


def _rounded(x, scale, fmt):
    """x to the nearest multiple of the format's step at its size, ties to the even one."""
    y = x / scale
    step = torch.ones_like(y)
    if fmt == "e4m3":
        step = torch.exp2((torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))) - 3)
    return torch.clamp(torch.round(y / step) * step, -LARGEST[fmt], LARGEST[fmt]) * scale


def _sequence(st, pages, scale, s, h, n):
    """The first n tokens of a head, as values, and the scale of each."""
    block = st["case"]["block"]
    page = st["table"][s, h, :-(-n // block)].long()
    sc = scale[page].double().repeat_interleave(block)[:n]
    return _decoded(pages[page].reshape(-1, D)[:n], st["case"]["format"]) * sc[:, None], sc


def exact(case, seed):
    st = prepare(case, seed)
    hq, hkv, fmt, op, block = (case[x] for x in ("q_heads", "kv_heads", "format", "op", "block"))
    lens, new, group = _head_lens(case), _new(case), hq // hkv
    pairs = [(s, h) for s in range(lens.shape[0]) for h in range(hkv)]
    if op == "attn":
        cu = _cu(new)
        out = torch.zeros((st["total"], hq, D), dtype=torch.float64, device=DEV)
        lse = torch.zeros((hq, st["total"]), dtype=torch.float64, device=DEV)
        weight = torch.zeros(st["weight"].shape, dtype=torch.float64, device=DEV) if "weight" in st else None
        for s, h in pairs:
            n, m, rows = int(lens[s, h]), int(new[s]), slice(int(cu[s]), int(cu[s + 1]))
            if weight is not None:
                weight[s, h, :n] = st["weight"][s, h, :n].double()
            if not m:
                continue
            k, v = (_sequence(st, st[x + "_pages"], st[x + "_scale"], s, h, n)[0] for x in "kv")
            q = st["q"][rows, h * group:(h + 1) * group].double().reshape(m * group, D)
            z = q @ k.T / math.sqrt(D)
            sees = (n - m + 1 + torch.arange(m, device=DEV)).repeat_interleave(group)
            hidden = torch.arange(n, device=DEV) >= sees[:, None]
            z = z.masked_fill(hidden, -math.inf)
            total = torch.logsumexp(z, 1)
            p = torch.exp(z - total[:, None]).masked_fill(hidden, 0.0)
            out[rows, h * group:(h + 1) * group] = (p @ v).view(m, group, D)
            lse[h * group:(h + 1) * group, rows] = total.view(m, group).T
            if weight is not None:
                weight[s, h, :n] += p.sum(0)
        return dict(out=out, lse=lse) | (dict(weight=weight) if weight is not None else {})
    back = _read_back(case)
    cu, new_cu = _cu(back), _cu(new)
    got = {x: torch.zeros((int(back.sum()), hkv, D), dtype=torch.float64, device=DEV) for x in "kv"}
    if op == "evict":
        keep = _keep(case)
        got |= dict(lens=torch.zeros(lens.shape, dtype=torch.int32, device=DEV), weight=torch.zeros(st["to_weight"].shape, dtype=torch.float64, device=DEV),
                    kept=torch.zeros(st["kept"].shape, dtype=torch.int32, device=DEV))
    for s, h in pairs:
        n = int(lens[s, h])
        if op == "evict":
            w = st["weight"][s, h, :n].double().cpu().numpy()
            left = min(n, max(int(keep[s, h]), SINK + RECENT))
            got["lens"][s, h] = left
            stays = np.zeros(n, bool)
            stays[:SINK] = stays[max(0, n - RECENT):] = True
            rest = np.flatnonzero(~stays)
            stays[rest[np.lexsort((rest, -w[rest]))][:left - int(stays.sum())]] = True
            at = np.flatnonzero(stays)[:left]
            got["kept"][s, h, :left] = torch.from_numpy(at.astype(np.int32)).to(DEV)
            got["weight"][s, h, :left] = torch.from_numpy(w[at]).to(DEV)
        for x in "kv":
            value, sc = _sequence(st, st[x + "_pages"], st[x + "_scale"], s, h, n)
            if op == "append":
                fresh = st[x][int(new_cu[s]):int(new_cu[s + 1]), h].double()[max(0, int(new[s]) - n):]
                start = n - fresh.shape[0]
                first = start // block * block                                 # pages from here on are written to
                value[start:] = fresh
                value[first:] = _paged(value[first:], fmt, block, float(sc[first]) if first < start and len(fresh) else 0.0, len(fresh) > 0)
            if op == "evict":
                value = _paged(value[torch.from_numpy(at).to(DEV)], fmt, block, 0.0, True)
            count = min(int(back[s]), value.shape[0])
            if count:
                got[x][int(cu[s + 1]) - count:int(cu[s + 1]), h] = value[value.shape[0] - count:]
    return got


def _paged(value, fmt, block, first_scale, written):
    """Values as pages hold them; the first page has a scale already, which does not shrink."""
    if not written or not value.shape[0]:
        return value
    n = value.shape[0]
    pages = torch.nn.functional.pad(value, (0, 0, 0, -n % block)).view(-1, block, D)
    sc = [_smallest(float(a), fmt) for a in pages.abs().amax((1, 2)).cpu()]
    sc[0] = max(sc[0], first_scale)
    sc = torch.tensor(sc, dtype=torch.float64, device=DEV)[:, None, None]
    return _rounded(pages, sc, fmt).view(-1, D)[:n]
