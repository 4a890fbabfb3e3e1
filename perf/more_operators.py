"""Serving on a paged KV cache beyond one token a sequence, as measured cases: block tables and slot
maps made on the GPU from request lengths, attention for trees of drafted tokens and the move that keeps an
accepted path, attention with a sliding window and a few first tokens that stay visible.

`run` computes them in plain torch, or, where `own` is true, through paper_2510_02613_b200.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "e4m3": 1}
MOST_FLOPS = 600e9    # of a drawn case, a little above the largest listed one
MOST_BYTES = 0.8e9


def listed():
    return [
        # a decode step of 64 sequences: each has one new token, every sixteenth needs a block for it
        dict(name="extend_64_decode", op="extend", seqs=64, lo=500, hi=2750, add_lo=1, add_hi=1, block=16, back=0.0),
        # a full batch: prompt pieces of up to 127 tokens, a fifth of the sequences give drafted tokens back
        dict(name="extend_1021_mixed", op="extend", seqs=1021, lo=0, hi=2750, add_lo=1, add_hi=127, block=16, back=0.2),
        # the accepted paths of 16 trees of 26 drafted tokens, four layers of a rank with 4 KV heads
        dict(name="keep_16_of_26", op="keep", seqs=16, nodes=26, most=5, layers=4, lo=26, hi=300, block=16, hkv=4, hd=128, kv="bf16", hm=False),
        # a large batch over the layers of a whole model, e4m3 with its scales, blocks [head][token]
        dict(name="keep_128_of_64_e4m3", op="keep", seqs=128, nodes=64, most=8, layers=24, lo=64, hi=100, block=16, hkv=4, hd=128, kv="e4m3", hm=True),
        # one sequence checks 8 drafted tokens on one of four tensor-parallel ranks of the large workload: latency
        dict(name="tree_1x8", op="tree", seqs=1, nodes_lo=8, nodes_hi=8, lo=2375, hi=2375, hq=8, hkv=1, hd=128, block=16, kv="bf16", io="bf16", hm=False),
        # 16 sequences with trees of 20 to 26 nodes on 32 query and 4 KV heads, f16, blocks [head][token]
        dict(name="tree_16x26_f16_hm", op="tree", seqs=16, nodes_lo=20, nodes_hi=26, lo=26, hi=2750, hq=32, hkv=4, hd=128, block=16, kv="f16", io="f16", hm=True),
        # every query head with a KV head of its own, an e4m3 cache, 5 to 13 nodes
        dict(name="tree_48x13_e4m3", op="tree", seqs=48, nodes_lo=5, nodes_hi=13, lo=13, hi=2750, hq=16, hkv=16, hd=128, block=16, kv="e4m3", io="bf16", hm=False),
        # wide trees over long contexts: bound by the products
        dict(name="tree_8x64_long", op="tree", seqs=8, nodes_lo=64, nodes_hi=64, lo=15000, hi=16411, hq=32, hkv=4, hd=128, block=16, kv="bf16", io="bf16", hm=False),
        # a decode step of 64 sequences, most of them longer than the window
        dict(name="window_64_decode", op="window", seqs=64, q_lo=1, q_hi=1, long=0, lo=100, hi=8192, window=1024, sinks=4, hq=32, hkv=4, hd=128, block=16, kv="bf16", io="bf16", hm=False),
        # a larger one with an e4m3 cache and a wide window
        dict(name="window_128_decode_e4m3", op="window", seqs=128, q_lo=1, q_hi=1, long=0, lo=1, hi=16384, window=4095, sinks=4, hq=16, hkv=2, hd=128, block=16, kv="e4m3", io="bf16", hm=False),
        # pieces of two prompts among 30 decoding sequences, f16, blocks [head][token]
        dict(name="window_mixed_f16_hm", op="window", seqs=32, q_lo=1, q_hi=1, long=2, long_lo=900, long_hi=1500, lo=1500, hi=6000, window=512, sinks=1, hq=32, hkv=4, hd=128, block=16, kv="f16", io="f16", hm=True),
        # a piece of 8192 tokens of one long prompt: bound by the products
        dict(name="window_prompt_8192", op="window", seqs=1, q_lo=1, q_hi=1, long=1, long_lo=8192, long_hi=8192, lo=12345, hi=12345, window=4096, sinks=4, hq=32, hkv=4, hd=128, block=16, kv="bf16", io="bf16", hm=False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("extend", "keep", "tree", "tree", "tree", "window", "window", "window"))
    block, hm = rng.choice((8, 16, 16, 32, 64)), rng.random() < 0.5
    if op == "extend":
        seqs = _log(rng, 1, 4096)
        hi = _log(rng, 1, 5000)
        add_hi = _log(rng, 1, max(1, 65536 // seqs))
        return dict(op=op, seqs=seqs, lo=rng.randint(0, hi), hi=hi, add_lo=rng.randint(1, add_hi), add_hi=add_hi, block=block,
                    back=rng.choice((0.0, 0.1, 0.5)))
    kv = rng.choice(("bf16", "f16", "e4m3"))
    hkv, hd = rng.choice((1, 2, 4, 8, 16)), rng.choice((32, 64, 128, 128, 128, 256))
    if op == "keep":
        nodes, lo = rng.randint(2, 64), rng.randint(1, 300)
        c = dict(op=op, seqs=_log(rng, 1, 256), nodes=nodes, most=rng.randint(1, min(nodes, 9)), layers=_log(rng, 1, 64), lo=nodes + lo,
                 hi=nodes + lo + rng.randint(0, 200), block=block, hkv=hkv, hd=hd, kv=kv, hm=hm)
        while c["seqs"] * c["hi"] * c["layers"] * 2 * hkv * hd * SIZE[kv] > 500e6:
            c["layers"], c["seqs"] = max(1, c["layers"] // 2), max(1, c["seqs"] * 3 // 4)
        return c
    io = rng.choice(("bf16", "f16")) if kv == "e4m3" else kv
    c = dict(op=op, seqs=_log(rng, 1, 128), hq=hkv * rng.choice((1, 2, 4, 5, 8)), hkv=hkv, hd=hd, block=block, kv=kv, io=io, hm=hm)
    if op == "tree":
        hi = _log(rng, 1, 128)
        c.update(nodes_lo=rng.randint(1, hi), nodes_hi=hi)
        top = _log(rng, hi, 32768)
        c.update(lo=rng.randint(hi, top), hi=top)
    else:
        c.update(q_lo=1, q_hi=rng.choice((1, 1, 1, 4)), long=0, window=_log(rng, 1, 8192), sinks=rng.choice((0, 1, 4, 4, 16, 100)))
        if rng.random() < 0.5:
            hi = _log(rng, 2, 8192)
            c.update(seqs=min(c["seqs"], 32), long_lo=rng.randint(1, hi), long_hi=hi)
            c["long"] = rng.randint(1, min(4, c["seqs"]))
        least = max(c["q_hi"], c.get("long_hi", 0))
        top = _log(rng, least, 32768)
        c.update(lo=rng.randint(least, top), hi=top)
    while True:
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and c["seqs"] * c["hi"] * 2 * hkv * hd * 4 <= 8e9:
            return c
        if c["seqs"] > 1:
            c["seqs"] = max(1, c["seqs"] // 2)
            if c.get("long"):
                c["long"] = min(c["long"], c["seqs"])
        else:
            c["hkv"] = hkv = max(1, c["hkv"] // 2)
            c["hq"] = max(c["hkv"], c["hq"] // 2 // c["hkv"] * c["hkv"])


# ---- inputs -------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 6151 + 29)


def _cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _lens(c):
    """Lengths spread evenly over the range, the new tokens included (their order is drawn)."""
    return np.linspace(c["lo"], c["hi"], c["seqs"]).astype(np.int64)


def _counts(c):
    """Query tokens of each sequence."""
    if c["op"] == "tree":
        return np.linspace(c["nodes_lo"], c["nodes_hi"], c["seqs"]).astype(np.int64)
    n = np.linspace(c["q_lo"], c["q_hi"], c["seqs"]).astype(np.int64)
    if c["long"]:
        n[: c["long"]] = np.linspace(c["long_lo"], c["long_hi"], c["long"]).astype(np.int64)
    return n


def _two_to(k):
    return ((k.clamp(min=-126) + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes and scale bytes of vectors along the last axis: the smallest power of two 2^k with
    amax <= 448 * 2^k, e4m3 rounded to nearest even."""
    x = x.float()
    amax = x.abs().amax(-1)
    mantissa, e = torch.frexp(amax)
    k = torch.where(amax == 0, torch.zeros_like(e), (e - 9 + (mantissa > 0.875).int()).clamp(min=-126))
    return (x * _two_to(-k)[..., None]).to(torch.float8_e4m3fn), (k + 127).to(torch.uint8)


def _arena(c, g, layers, pool):
    """K and V pools of the layers, as bytes, and the scale bytes of an e4m3 cache."""
    inner = (c["hkv"], c["block"]) if c["hm"] else (c["block"], c["hkv"])
    shape = (layers, 2, pool) + inner + (c["hd"],)
    arena = torch.empty(shape, dtype=TYPES[c["kv"]], device="cuda")
    scales = torch.empty(shape[:-1], dtype=torch.uint8, device="cuda") if c["kv"] == "e4m3" else None
    for i in range(layers):
        for j in range(2):
            x = torch.randn(shape[2:], generator=g, device="cuda")
            if scales is None:
                arena[i, j] = x.to(TYPES[c["kv"]])
            else:
                arena[i, j], scales[i, j] = _quantise(x)
    return arena.view(torch.uint8), scales


def _tables(c, host, lens, width, skip=None):
    """A table of blocks of their own for every sequence (-1 where it has none); skip: per sequence the blocks
    [a, b) that it no longer holds."""
    held = [[j for j in range(-(-int(n) // c["block"])) if skip is None or not skip[i][0] <= j < skip[i][1]] for i, n in enumerate(lens)]
    pool = sum(map(len, held)) + 3
    ids = host.permutation(pool).astype(np.int32)
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for i, cols in enumerate(held):
        table[i, cols] = ids[at:at + len(cols)]
        at += len(cols)
    return table, pool, ids[at:]


def _tree_masks(host, counts, words):
    """Ancestors (and itself) of each node of random trees, bit k of a row: node k."""
    rows = np.zeros((int(counts.sum()), words * 32), bool)
    at = 0
    for n in counts:
        for i in range(int(n)):
            if i:
                rows[at + i] = rows[at + host.randint(max(0, (i - 1) // 3 - 2), i)]   # wide trees: a few children a node
            rows[at + i, i] = True
        at += int(n)
    bits = np.packbits(rows.reshape(-1, words, 4, 8), axis=-1, bitorder="little")[..., 0]
    return bits.reshape(-1, words * 4).view("<i4")


def prepare(case, seed):
    c, g = case, _gen(seed)
    host = np.random.RandomState(seed % (1 << 31))
    n, b = c["seqs"], c["block"]
    lens = host.permutation(_lens(c)).astype(np.int32)
    s = dict(case=c)
    if c["op"] == "extend":
        add = host.randint(c["add_lo"], c["add_hi"] + 1, n).astype(np.int32)
        back = host.rand(n) < c["back"]
        add[back] = -np.minimum(lens[back], add[back])
        width = -(-(int(lens.max()) + c["add_hi"]) // b)
        table, pool, _ = _tables(c, host, lens, width)
        # the lists have the same room whatever the lengths of a step
        more = n * (-(-c["add_hi"] // b) + 1)
        free = np.full(more + int(-(-_lens(c) // b).sum()), -1, np.int32)
        free[:more] = pool + host.permutation(more)
        s.update(lens=_cuda(lens), add=_cuda(add), table=_cuda(table), free=_cuda(free), n_free=_cuda(np.array([more], np.int32)), pool=pool + more)
        tokens = n * c["add_hi"] + 5
        s.update(lens_out=torch.empty_like(s["lens"]), n_free_out=torch.empty_like(s["n_free"]), q_start=torch.empty(n + 1, dtype=torch.int32, device="cuda"),
                 slots=torch.empty(tokens, dtype=torch.int64, device="cuda"))
        return s
    if c["op"] == "keep":
        width = -(-c["hi"] // b)
        table, pool, _ = _tables(c, host, lens, width)
        count = host.randint(1, c["most"] + 1, n).astype(np.int32)
        accepted = np.full((n, c["most"]), -1, np.int32)
        for i, m in enumerate(count):
            # the root and a rising path; a node in the way of a shorter one's new place is that node itself, so that
            # the same pass can be made again
            far = host.permutation(np.arange(m, c["nodes"]))[: m - 1]
            m = count[i] = 1 + len(far)
            accepted[i, :m] = np.concatenate([[0], np.sort(far)])
        s.update(lens=_cuda(lens), table=_cuda(table), accepted=_cuda(accepted), count=_cuda(count), pool=pool,
                 q_start=_cuda(np.arange(n + 1, dtype=np.int32) * c["nodes"]), change=torch.empty(n, dtype=torch.int32, device="cuda"))
        s["arena"], s["scales"] = _arena(c, g, c["layers"], pool)
        return s
    counts = host.permutation(_counts(c)) if c["op"] == "tree" else _counts(c)
    skip = None
    if c["op"] == "window":   # blocks that the window has left behind are given back
        first = np.maximum(lens - counts + 1 - c["window"], 0)
        skip = [(-(-c["sinks"] // b), int(f) // b) for f in first]
    table, pool, _ = _tables(c, host, lens, -(-c["hi"] // b), skip)
    starts = np.zeros(n + 1, np.int32)
    starts[1:] = np.cumsum(counts)
    tokens = int(starts[-1])
    s.update(host_lens=lens.tolist(), host_counts=counts.tolist(), lens=_cuda(lens), table=_cuda(table), pool=pool, q_start=_cuda(starts),
             max_q=int(counts.max()))
    s["arena"], s["scales"] = _arena(c, g, 1, pool)
    s["q"] = (torch.randn((tokens, c["hq"], c["hd"]), generator=g, device="cuda") * 1.5).to(TYPES[c["io"]])
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((tokens, c["hq"]), device="cuda")
    if c["op"] == "tree":
        s["mask"] = _cuda(_tree_masks(host, counts, -(-c["nodes_hi"] // 32)))
    return s


# ---- one pass -----------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    if own:
        return {"extend": _own_extend, "keep": _own_keep, "tree": _own_tree, "window": _own_window}[op](state)
    return {"extend": _extend, "keep": _keep, "tree": _attend, "window": _attend}[op](state)


def _cache(s):
    """The handle on the arena, made once as a serving program would."""
    if "cache" not in s:
        import paper_2510_02613_b200 as E
        c = s["case"]
        arena = s["arena"] if "arena" in s else torch.empty(2 * s["pool"] * c["block"] * 8 * 2, dtype=torch.uint8, device="cuda")
        s["cache"] = E.KvCache(arena, n_layers=c.get("layers", 1), num_blocks=s["pool"], block_tokens=c["block"], n_heads=c.get("hkv", 1),
                               head_dim=c.get("hd", 8), kv_type=c.get("kv", "bf16"), scales=s.get("scales"), head_major=c.get("hm", False))
    return s["cache"]


def _own_extend(s):
    _cache(s).extend(s["lens"], s["add"], s["table"], s["free"], s["n_free"], s["q_start"], s["slots"], s["lens_out"], s["n_free_out"])
    return s["lens_out"], s["table"], s["free"], s["n_free_out"], s["q_start"], s["slots"]


def _own_keep(s):
    _cache(s).keep(s["table"], s["lens"], s["q_start"], s["accepted"], s["count"], s["change"])
    return _held(s)


def _own_tree(s):
    cache, c = _cache(s), s["case"]
    if "work" not in s:
        n = cache.attend_tree_workspace_bytes(c["seqs"], s["q"].shape[0], s["max_q"], c["hq"], s["table"].shape[1])
        s["work"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    cache.attend_tree(0, s["q"], s["out"], s["table"], s["lens"], s["q_start"], s["mask"], s["max_q"], lse=s["lse"], workspace=s["work"])
    return s["out"], s["lse"]


def _own_window(s):
    cache, c = _cache(s), s["case"]
    if "work" not in s:
        n = cache.attend_window_workspace_bytes(c["seqs"], s["q"].shape[0], s["max_q"], c["hq"], s["table"].shape[1], c["window"], c["sinks"])
        s["work"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    cache.attend_window(0, s["q"], s["out"], s["table"], s["lens"], s["q_start"], s["max_q"], c["window"], c["sinks"], lse=s["lse"],
                        workspace=s["work"])
    return s["out"], s["lse"]


def _extend(s):
    """Blocks are given in the order of the sequences from the end of the free list, behind which those given back
    come first; every sequence of these cases gets what it needs."""
    b, n = s["case"]["block"], s["case"]["seqs"]
    lens, add, table, free = s["lens"].long(), s["add"].long(), s["table"], s["free"]
    after = (lens + add).clamp(min=0)
    had, has = (lens + b - 1) // b, (after + b - 1) // b
    column = torch.arange(table.shape[1], device="cuda")
    gone = (column >= has[:, None]) & (column < had[:, None])
    new = (column >= had[:, None]) & (column < has[:, None])
    order = gone.flatten().long().cumsum(0) - 1
    at = s["n_free"].long() + order
    at = torch.where(gone.flatten(), at, free.numel())   # a place behind the list for what stays
    free.copy_(torch.cat([free, free[:1]]).scatter(0, at, table.flatten())[:-1])
    top = s["n_free"].long() + gone.sum()
    order = (new.flatten().long().cumsum(0) - 1).view_as(table)
    table.copy_(torch.where(new, free[(top - 1 - order).clamp(min=0)], table))
    s["lens_out"].copy_(after)
    s["n_free_out"].copy_(top - new.sum())
    s["q_start"][0] = 0
    s["q_start"][1:] = add.clamp(min=0).cumsum(0)
    i = torch.arange(s["slots"].numel(), device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), i, right=True).clamp(max=n - 1)
    place = lens[seq] + i - s["q_start"].long()[seq]
    inside = i < s["q_start"][-1]
    place = torch.where(inside, place, 0)
    s["slots"].copy_(torch.where(inside, table[seq, place // b].long() * b + place % b, -1))
    return s["lens_out"], table, free, s["n_free_out"], s["q_start"], s["slots"]


def _at(c, slots):
    """Index of token slots in a (pool, ...) tensor."""
    block, off = slots // c["block"], slots % c["block"]
    return (block, slice(None), off) if c["hm"] else (block, off)


def _held(s):
    """The sequences' change of length and what the cache holds: 16-bit values, or e4m3 codes and their scales."""
    codes = s["arena"].view(TYPES[s["case"]["kv"]])
    return (s["change"], codes) + ((s["scales"].view(torch.float8_e8m0fnu),) if s["scales"] is not None else ())


def _keep(s):
    c = s["case"]
    at = torch.arange(c["most"], device="cuda")
    start = s["lens"].long() - (s["q_start"][1:] - s["q_start"][:-1]).long()
    s["change"].copy_(s["count"] - (s["q_start"][1:] - s["q_start"][:-1]))
    real = at < s["count"][:, None]
    source = torch.where(real, start[:, None] + s["accepted"], start[:, None])   # the root stays where it is
    target = torch.where(real, start[:, None] + at, start[:, None])
    source, target = ((s["table"].long().gather(1, x // c["block"]) * c["block"] + x % c["block"]).flatten() for x in (source, target))
    for x in (s["arena"], s["scales"]):
        if x is not None:
            for pool in x.flatten(0, 1):
                pool[_at(c, target)] = pool[_at(c, source)]
    return _held(s)


def _rows(s, i, slots):
    """K (i = 0) or V (i = 1) vectors of token slots in 32 bits: [slots, heads, hd]."""
    c = s["case"]
    x = s["arena"].view(TYPES[c["kv"]] if c["kv"] != "e4m3" else torch.uint8)[0, i][_at(c, slots)]
    if c["kv"] == "e4m3":
        byte = s["scales"][0, i][_at(c, slots)].int()
        x = x.view(torch.float8_e4m3fn).float() * _two_to(byte - 127)[..., None]
    return x.float()


def _attend(s):
    c = s["case"]
    hkv, hd, b = c["hkv"], c["hd"], c["block"]
    first = 0
    for i, (length, n) in enumerate(zip(s["host_lens"], s["host_counts"])):
        context = length - n
        if c["op"] == "tree":
            token = torch.arange(length, device="cuda")
        else:
            start = max(0, context + 1 - c["window"])
            token = torch.cat([torch.arange(min(c["sinks"], start), device="cuda"), torch.arange(start, length, device="cuda")])
        slots = s["table"][i].long()[token // b] * b + token % b
        k, v = _rows(s, 0, slots), _rows(s, 1, slots)
        step = max(1, min(n, (1 << 28) // (c["hq"] * len(token))))
        for t in range(0, n, step):
            at = slice(first + t, first + min(n, t + step))
            row = torch.arange(t, min(n, t + step), device="cuda")
            if c["op"] == "tree":
                node = torch.arange(n, device="cuda")
                bits = (s["mask"][at][:, node // 32] >> (node % 32).int()) & 1
                seen = torch.cat([torch.ones((len(row), context), dtype=torch.bool, device="cuda"), bits.bool()], 1)
            else:
                place = context + row[:, None]
                seen = (token <= place) & ((token < c["sinks"]) | (token > place - c["window"]))
            q = s["q"][at].float().reshape(len(row), hkv, -1, hd) * hd ** -0.5
            score = torch.einsum("nhgd,thd->nhgt", q, k).masked_fill_(~seen[:, None, None], float("-inf"))
            top = score.amax(-1, keepdim=True)
            safe = torch.where(torch.isinf(top), 0.0, top)
            score = torch.exp(score.sub_(safe))
            total = score.sum(-1, keepdim=True)
            o = torch.einsum("nhgt,thd->nhgd", score, v)
            s["out"][at] = torch.where(total > 0, o / total, 0.0).reshape(len(row), -1, hd).to(s["out"].dtype)
            s["lse"][at] = (torch.log(total) + safe)[..., 0].reshape(len(row), -1)
        first += n
    return s["out"], s["lse"]


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    c = case
    if c["op"] == "extend":
        new = c["seqs"] * (1 - c["back"]) * (c["add_lo"] + c["add_hi"]) / 2
        # lengths and changes read, lengths and starts written; the whole slot map; a block id read and written a block
        return {"bytes": int(c["seqs"] * 16 + (c["seqs"] * c["add_hi"] + 5) * 8 + 2 * 4 * new / c["block"]), "flops": 0}
    if c["op"] == "keep":
        moved = c["seqs"] * (c["most"] - 1) / 2   # of 1 to `most` accepted tokens all but the root
        per = 2 * c["layers"] * c["hkv"] * (c["hd"] * SIZE[c["kv"]] + (1 if c["kv"] == "e4m3" else 0))
        return {"bytes": int(2 * moved * per + c["seqs"] * (4 * c["most"] + 24)), "flops": 0}
    # lengths and query tokens are paired anew with every seed: by their means
    lens, counts = _lens(c), _counts(c)
    per = 2 * c["hkv"] * (c["hd"] * SIZE[c["kv"]] + (1 if c["kv"] == "e4m3" else 0))
    tokens = pairs = 0
    for n in counts:
        for length in lens[:: max(1, len(lens) // 8)]:
            share = 1 / len(lens[:: max(1, len(lens) // 8)])
            if c["op"] == "tree":
                tokens += share * length
                pairs += share * n * (length - n + math.log(n + 1, 2) + 1)
            else:
                place = np.arange(length - n, length)
                seen = np.minimum(place + 1, c["window"]) + np.minimum(c["sinks"], np.maximum(0, place + 1 - c["window"]))
                start = max(0, length - n + 1 - c["window"])
                tokens += share * (length - start + min(c["sinks"], start))
                pairs += share * int(seen.sum())
    rows = int(counts.sum()) * c["hq"]
    return {"bytes": int(tokens * per + rows * (2 * c["hd"] * SIZE[c["io"]] + 4)), "flops": int(4 * c["hq"] * c["hd"] * pairs)}


# ---- the definitions in 64 bits -----------------------------------------------------------------


def _vectors(s, i, head, blocks, positions):
    """Vectors [positions, hd] of one head in 64 bits."""
    c = s["case"]
    block, off = blocks[torch.div(positions, c["block"], rounding_mode="floor")], positions.remainder(c["block"])
    at = (0, i, block, head, off) if c["hm"] else (0, i, block, off, head)
    x = s["arena"].view(TYPES[c["kv"]])[at].double()
    return x if s["scales"] is None else x * torch.exp2(s["scales"][at].double() - 127)[:, None]


def exact(case, seed):
    c = case
    if c["op"] == "extend":
        return None   # whole numbers
    s = prepare(case, seed)
    if c["op"] == "keep":
        table, lens, accepted = s["table"].tolist(), s["lens"].tolist(), s["accepted"].tolist()
        pools = [x for x in (s["arena"].view(TYPES[c["kv"]]), s["scales"]) if x is not None]
        pools = [(x.transpose(3, 4) if c["hm"] else x) for x in pools]   # a view: (layer, K or V, block, offset, head)
        for i, m in enumerate(s["count"].tolist()):
            for j in range(1, m):
                at, to = (divmod(lens[i] - c["nodes"] + k, c["block"]) for k in (accepted[i][j], j))
                for x in pools:
                    x[:, :, table[i][to[0]], to[1]] = x[:, :, table[i][at[0]], at[1]]
        kept = (s["count"] - c["nodes"], s["arena"].view(TYPES[c["kv"]]).double())
        return kept if s["scales"] is None else kept + (torch.exp2(s["scales"].double() - 127),)
    q = s["q"].double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], float("-inf"), dtype=torch.float64, device="cuda")
    group, first = c["hq"] // c["hkv"], 0
    for i in range(c["seqs"]):
        length, n = s["host_lens"][i], s["host_counts"][i]
        blocks = s["table"][i].long()
        for t in range(0, n, 1024):
            m = min(1024, n - t)
            position = length - n + t + torch.arange(m, device="cuda")
            if c["op"] == "tree":
                tokens = torch.arange(length, device="cuda")
                bit = torch.arange(32, device="cuda", dtype=torch.int32)
                bits = ((s["mask"][first + t:first + t + m, :, None] >> bit) & 1).flatten(1)[:, :n].bool()
                hidden = torch.cat([torch.zeros((m, length - n), dtype=torch.bool, device="cuda"), ~bits], 1)
            else:
                low = max(0, length - n + t - c["window"] + 1)
                sinks = min(c["sinks"], low)
                tokens = torch.arange(sinks + length - low, device="cuda")
                tokens = torch.where(tokens < sinks, tokens, tokens - sinks + low)
                behind = (tokens[None] <= position[:, None] - c["window"]) & (tokens[None] >= c["sinks"])
                hidden = behind | (tokens[None] > position[:, None])
            for h in range(c["hkv"]):
                k, v = _vectors(s, 0, h, blocks, tokens), _vectors(s, 1, h, blocks, tokens)
                for j in range(h * group, (h + 1) * group):
                    score = (q[first + t:first + t + m, j] @ k.t() / math.sqrt(c["hd"])).masked_fill(hidden, float("-inf"))
                    lse[first + t:first + t + m, j] = torch.logsumexp(score, -1)
                    weight = torch.softmax(score, -1)
                    out[first + t:first + t + m, j] = torch.where(hidden.all(-1)[:, None], 0.0, weight @ v)
        first += n
    return out, lse


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(8)]:
        print(c, work(c))
