"""The serving operators on the library's arenas, as measured cases: writing and reading a paged KV
cache that is held in 16 bits or in e4m3 with a power-of-two scale per head vector, decode
attention for a batch that shares a prefix, and a whole mixture-of-experts layer for a few tokens.

`run` computes them in plain torch, or, where `own` is true, through paper_2510_02613_b200.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}


def listed():
    return [
        # one decode step of a batch of 64 sequences writes its new keys and values (16 heads x 128, as the
        # fine-grained workload): a call of a few microseconds
        dict(name="append_64_e4m3", op="append", tokens=64, pool=512, block=16, heads=16, hd=128, kv="e4m3", io="bf16", hm=False),
        # a chunk of prompts written at once
        dict(name="append_8191_e4m3", op="append", tokens=8191, pool=1024, block=16, heads=16, hd=128, kv="e4m3", io="bf16", hm=False),
        # one sequence of the workloads' middle length read back on a rank with one KV head, blocks [head][token]
        dict(name="gather_2375_e4m3_hm", op="gather", tokens=2375, pool=512, block=16, heads=1, hd=128, kv="e4m3", io="bf16", hm=True),
        # the whole 64k-token cache of the fine-grained workload, one layer
        dict(name="gather_65536_e4m3", op="gather", tokens=65536, pool=4608, block=16, heads=16, hd=128, kv="e4m3", io="bf16", hm=False),
        # one sequence, no prefix, on one of four tensor-parallel ranks of the large workload: latency
        dict(name="attend_1_own2375", op="attend", seqs=1, qlen=1, hq=8, hkv=1, hd=128, prefix=0, lo=2375, hi=2375, block=16, kv="bf16", io="bf16", hm=False),
        # 48 requests with a common 2000-token prompt and 500 to 750 tokens of their own (32 query, 4 KV heads)
        dict(name="attend_48_prefix2000", op="attend", seqs=48, qlen=1, hq=32, hkv=4, hd=128, prefix=2000, lo=500, hi=750, block=16, kv="bf16", io="bf16", hm=False),
        # every query head with a KV head of its own, an e4m3 cache, an odd prefix that ends inside a block
        dict(name="attend_32_prefix8199_e4m3", op="attend", seqs=32, qlen=1, hq=16, hkv=16, hd=128, prefix=8199, lo=1, hi=750, block=16, kv="e4m3", io="bf16", hm=False),
        # four drafted tokens of 16 sequences checked at once, f16, blocks [head][token]
        dict(name="attend_16x4_prefix4096_hm", op="attend", seqs=16, qlen=4, hq=32, hkv=4, hd=128, prefix=4096, lo=4, hi=2750, block=16, kv="f16", io="f16", hm=True),
        # a large batch over a very long shared document: bound by the products, not by memory
        dict(name="attend_128_prefix65536", op="attend", seqs=128, qlen=1, hq=32, hkv=4, hd=128, prefix=65536, lo=500, hi=750, block=16, kv="bf16", io="bf16", hm=False),
        # one token through the fine-grained layer: 6 of 64 experts and 2 shared ones
        dict(name="moe_1_fine", op="moe", tokens=1, d=2048, f=1408, experts=64, held=64, shared=2, k=6, w="bf16", io="bf16", fused=False),
        # 16 tokens on one of eight ranks of the wide FP8 layer: 32 of 256 experts and the shared one
        dict(name="moe_16_wide_e4m3", op="moe", tokens=16, d=7168, f=2048, experts=256, held=32, shared=1, k=8, w="e4m3", io="bf16", fused=False),
        # the most tokens a call takes, all experts of the large workload's layer, gate and up fused
        dict(name="moe_64_large_w13", op="moe", tokens=64, d=2048, f=768, experts=128, held=128, shared=0, k=8, w="bf16", io="bf16", fused=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "gather", "attend", "attend", "attend", "moe", "moe"))
    kv = rng.choice(("bf16", "f16", "e4m3", "e4m3"))
    io = rng.choice(("bf16", "f16")) if kv == "e4m3" else kv
    block, hm = rng.choice((8, 16, 16, 32, 64)), rng.random() < 0.5
    if op in ("append", "gather"):
        tokens = _log(rng, 1, 8192 if op == "append" else 65536)
        heads, hd = rng.choice((1, 2, 4, 8, 16)), rng.choice((32, 64, 128))
        if rng.random() < 0.2 and kv == "e4m3":
            io = "f32"
        pool = -(-tokens // block) + rng.randint(1, 64)
        return dict(op=op, tokens=tokens, pool=pool, block=block, heads=heads, hd=hd, kv=kv, io=io, hm=hm)
    if op == "attend":
        hkv, group = rng.choice((1, 2, 4, 8, 16)), rng.choice((1, 2, 4, 5, 8))
        hd = rng.choice((32, 64, 128, 128))
        seqs, qlen = _log(rng, 1, 128), rng.choice((1, 1, 1, 2, 4))
        prefix = rng.choice((0, 1)) * _log(rng, 1, 65536)
        hi = _log(rng, 1, 2750)
        lo = rng.randint(1, hi)
        while seqs * qlen * hkv * group * (prefix + hi) * hd > 128 * 32 * 66000 * 128:
            prefix, seqs = prefix // 2, max(1, seqs // 2)
        return dict(op=op, seqs=seqs, qlen=qlen, hq=hkv * group, hkv=hkv, hd=hd, prefix=prefix, lo=lo, hi=hi, block=block, kv=kv, io=io, hm=hm)
    w = rng.choice(("bf16", "f16", "e4m3"))
    d, f = 16 * _log(rng, 16, 448), 16 * _log(rng, 8, 128)
    experts = rng.choice((8, 60, 64, 128, 256))
    held = rng.choice((experts, -(-experts // 3), -(-experts // 8)))
    shared, k = rng.choice((0, 0, 1, 2)), rng.choice((1, 2, 4, 6, 8))
    while (held + shared) * 3 * d * f * SIZE[w] > 1_400_000_000:
        held = max(1, held // 2)
    return dict(op="moe", tokens=_log(rng, 1, 64), d=d, f=f, experts=experts, held=held, shared=shared, k=k, w=w,
                io=rng.choice(("bf16", "f16")) if w == "e4m3" else w, fused=w != "e4m3" and rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _two_to(k):
    """2^k in 32 bits, made of its bits: exact for every exponent that a scale has."""
    return ((k.clamp(min=-126) + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes and scale bytes of vectors along the last axis: the smallest power of two 2^k with
    amax <= 448 * 2^k (k >= -126; 0 for a zero vector), e4m3 rounded to nearest even.  A vector
    that is not finite: byte 255, codes 0."""
    x = x.float()
    amax = x.abs().amax(-1)
    mantissa, e = torch.frexp(amax)
    k = (e - 9 + (mantissa > 0.875).int()).clamp(min=-126)
    k = torch.where(amax == 0, torch.zeros_like(k), k)
    good = torch.isfinite(amax)
    k = torch.where(good, k, torch.zeros_like(k))
    x = torch.where(good[..., None], x, torch.zeros_like(x))
    codes = (x * _two_to(-k)[..., None]).to(torch.float8_e4m3fn)
    return codes, torch.where(good, k + 127, torch.full_like(k, 255)).to(torch.uint8)


def _pool(c):
    """Shapes of the K and V pools of one layer: codes and scale bytes."""
    inner = (c["heads"], c["block"]) if c["hm"] else (c["block"], c["heads"])
    return (2, c["pool"]) + inner


def prepare(case, seed):
    c, g = case, _gen(seed)
    host = np.random.RandomState(seed % (1 << 31))
    if c["op"] in ("append", "gather"):
        n, shape = c["tokens"], (c["tokens"], c["heads"], c["hd"])
        slots = torch.from_numpy(host.permutation(c["pool"] * c["block"])[:n].astype(np.int64))   # a decode step: one token each
        if c["op"] == "gather" or n > 256:   # a prompt or a sequence: whole blocks, in the order of its table
            blocks = host.permutation(c["pool"])[: -(-n // c["block"])].astype(np.int64)
            slots = torch.from_numpy((blocks[:, None] * c["block"] + np.arange(c["block"])).reshape(-1)[:n].copy())
        s = dict(case=c, slots=slots.cuda())
        old = _randn(g, _pool(c) + (c["hd"],), torch.float32 if c["kv"] == "e4m3" else TYPES[c["kv"]])
        if c["kv"] == "e4m3":
            codes, s["scales"] = _quantise(old)
            s["arena"] = codes.view(torch.uint8)
        else:
            s["arena"], s["scales"] = old.view(torch.uint8), None
        if c["op"] == "append":
            # keys have a few channels far larger than the others
            channel = torch.where(torch.rand(c["hd"], generator=g, device="cuda") < 0.05, 8.0, 1.0)
            s["k"] = (torch.randn(shape, generator=g, device="cuda") * channel).to(TYPES[c["io"]])
            s["v"] = _randn(g, shape, TYPES[c["io"]], 0.5)
        else:
            s["k"], s["v"] = (torch.empty(shape, dtype=TYPES[c["io"]], device="cuda") for _ in range(2))
        return s
    if c["op"] == "attend":
        n, b = c["seqs"], c["block"]
        lens = host.permutation(_lens(c)).astype(np.int32)
        need = [-(-int(x) // b) for x in lens]
        pre = -(-c["prefix"] // b)
        pool = pre + sum(need) + 3
        ids = host.permutation(pool).astype(np.int32)
        table = np.full((n, max(need)), -1, np.int32)
        at = pre
        for i, m in enumerate(need):
            table[i, :m] = ids[at:at + m]
            at += m
        s = dict(case=dict(c, pool=pool, heads=c["hkv"]), lens=torch.from_numpy(lens).cuda(), table=torch.from_numpy(table).cuda(),
                 prefix_table=torch.from_numpy(ids[:pre].copy()).cuda())
        shape = _pool(s["case"]) + (c["hd"],)
        kv = torch.randn(shape, generator=g, device="cuda")
        if c["kv"] == "e4m3":
            codes, s["scales"] = _quantise(kv)
            s["arena"] = codes.view(torch.uint8)
        else:
            s["arena"], s["scales"] = kv.to(TYPES[c["kv"]]).view(torch.uint8), None
        del kv
        s["q"] = _randn(g, (n, c["qlen"], c["hq"], c["hd"]), TYPES[c["io"]], 1.5)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((n, c["qlen"], c["hq"]), device="cuda")
        return s
    slots, d, f = c["held"] + c["shared"], c["d"], c["f"]
    m = d * f
    size = SIZE[c["w"]]
    weights = torch.empty(3 * slots * m * size, dtype=torch.uint8, device="cuda")
    w = weights.view(TYPES[c["w"]])
    step = 1 << 27
    for i in range(0, w.numel(), step):
        part = w[i:i + step]
        # bounded as trained weights are; e4m3 codes use their whole range, the scales bring them down
        scale = 100.0 if c["w"] == "e4m3" else 1.0 / math.sqrt(d)
        part.copy_((torch.randn(part.numel(), generator=g, device="cuda") * scale).clamp_(-4 * scale, 4 * scale))
    s = dict(case=c, arena=weights)
    if c["w"] == "e4m3":   # one fp32 scale per 128 x 128 block, behind the weights from the next multiple of 256
        blocks = -(-d // 128) * -(-f // 128)
        at = -(-weights.numel() // 256) * 256
        s["arena"] = torch.zeros(at + 3 * slots * blocks * 4, dtype=torch.uint8, device="cuda")
        s["arena"][:weights.numel()] = weights
        s["arena"][at:].view(torch.float32).copy_((0.5 + torch.rand(3 * slots * blocks, generator=g, device="cuda")) / (100 * math.sqrt(d)))
    table = np.full(c["experts"] + c["shared"], -1, np.int32)
    table[host.permutation(c["experts"])[:c["held"]]] = host.permutation(c["held"])
    table[c["experts"]:] = np.arange(c["held"], slots)
    s["slot_of_expert"] = torch.from_numpy(table).cuda()
    s["logits"] = torch.from_numpy(_logits(c, host)).cuda()
    s["x"] = _randn(g, (c["tokens"], d), TYPES[c["io"]])
    s["out"] = torch.empty_like(s["x"])
    s["ids"] = torch.empty((c["tokens"], c["k"]), dtype=torch.int32, device="cuda")
    s["weights"] = torch.empty((c["tokens"], c["k"]), device="cuda")
    return s


def _lens(c):
    """Own lengths spread evenly over the range (their order is drawn)."""
    return np.linspace(c["lo"], c["hi"], c["seqs"]).astype(np.int64)


def _logits(c, host):
    """Router logits: normal, with some experts more popular than others."""
    bias = 0.5 * host.standard_normal(c["experts"])
    return (host.standard_normal((c["tokens"], c["experts"])) + bias).astype(np.float32)


# ---- one pass -----------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "gather": _own_gather, "attend": _own_attend, "moe": _own_moe}[op](state)
    return {"append": _append, "gather": _gather, "attend": _attend, "moe": _moe}[op](state)


def _cache(s):
    """The handle on the arena, made once as a serving program would."""
    if "cache" not in s:
        import paper_2510_02613_b200 as E
        c = s["case"]
        s["cache"] = E.KvCache(s["arena"], n_layers=1, num_blocks=c["pool"], block_tokens=c["block"], n_heads=c["heads"],
                               head_dim=c["hd"], kv_type=c["kv"], scales=s["scales"], head_major=c["hm"])
    return s["cache"]


def _own_append(s):
    _cache(s).append(0, s["k"], s["v"], s["slots"])
    return _held(s)


def _own_gather(s):
    _cache(s).gather(0, s["slots"], s["k"], s["v"])
    return s["k"], s["v"]


def _own_attend(s):
    cache, c = _cache(s), s["case"]
    if "work" not in s:
        n = cache.attend_workspace_bytes(c["seqs"], c["qlen"], c["hq"], s["table"].shape[1], c["prefix"])
        s["work"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    cache.attend(0, s["q"], s["out"], s["table"], s["lens"], prefix_table=s["prefix_table"], prefix_len=c["prefix"], lse=s["lse"],
                 workspace=s["work"])
    return s["out"], s["lse"]


def _own_moe(s):
    c = s["case"]
    if "experts" not in s:
        import paper_2510_02613_b200 as E
        s["experts"] = E.ExpertArena(s["arena"], n_layers=1, n_slots=c["held"] + c["shared"], d_model=c["d"], d_ff=c["f"], w_type=c["w"],
                                     fused_w13=c["fused"])
        n = s["experts"].decode_workspace_bytes(c["tokens"], c["k"], c["experts"], c["shared"])
        s["work"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    s["experts"].decode(0, s["x"], s["logits"], c["k"], s["slot_of_expert"], s["out"], n_shared=c["shared"], ids_out=s["ids"],
                        weights_out=s["weights"], workspace=s["work"])
    return s["out"], s["ids"], s["weights"]


def _held(s):
    """What the cache holds: 16-bit values, or e4m3 codes and their scales."""
    c = s["case"]
    codes = s["arena"].view(TYPES[c["kv"]])
    return (codes, s["scales"].view(torch.float8_e8m0fnu)) if c["kv"] == "e4m3" else codes


def _at(c, slots):
    """Index of token slots in a (pool, ...) tensor, heads last but one."""
    block, off = slots // c["block"], slots % c["block"]
    return (block, slice(None), off) if c["hm"] else (block, off)


def _append(s):
    c = s["case"]
    arena = s["arena"].view(TYPES[c["kv"]]) if c["kv"] != "e4m3" else s["arena"]
    for i, x in enumerate((s["k"], s["v"])):
        if c["kv"] == "e4m3":
            codes, byte = _quantise(x)
            arena[i][_at(c, s["slots"])] = codes.view(torch.uint8)
            s["scales"][i][_at(c, s["slots"])] = byte
        else:
            arena[i][_at(c, s["slots"])] = x.float().to(TYPES[c["kv"]])
    return _held(s)


def _rows(s, i, slots):
    """K (i = 0) or V (i = 1) vectors of token slots in 32 bits: slots.shape + (heads, hd)."""
    c = s["case"]
    x = s["arena"].view(TYPES[c["kv"]]) if c["kv"] != "e4m3" else s["arena"]
    flat = slots.reshape(-1)
    x = x[i][_at(c, flat)]
    if c["kv"] == "e4m3":
        byte = s["scales"][i][_at(c, flat)].int()
        x = x.view(torch.float8_e4m3fn).float() * _two_to((byte - 127).clamp(max=127))[..., None]
        x = torch.where((byte == 255)[..., None], float("nan"), x)
    return x.float().reshape(slots.shape + x.shape[1:])


def _gather(s):
    t = TYPES[s["case"]["io"]]
    return _rows(s, 0, s["slots"]).to(t), _rows(s, 1, s["slots"]).to(t)


def _attend(s):
    c = s["case"]
    n, t, hkv, hd = c["seqs"], c["qlen"], c["hkv"], c["hd"]
    q = s["q"].float().reshape(n, t, hkv, -1, hd) * hd ** -0.5
    at = torch.arange(c["prefix"], device="cuda")
    slots = s["prefix_table"].long()[at // c["block"]] * c["block"] + at % c["block"]
    kp, vp = _rows(s, 0, slots), _rows(s, 1, slots)
    at = torch.arange(s["table"].shape[1] * c["block"], device="cuda")
    slots = s["table"].long()[:, at // c["block"]].clamp(min=0) * c["block"] + at % c["block"]
    ko, vo = _rows(s, 0, slots), _rows(s, 1, slots)
    last = s["lens"][:, None] - t + torch.arange(t, device="cuda")
    seen = at <= last[..., None]
    vo = vo * (at < s["lens"][:, None])[..., None, None]
    sp = torch.einsum("nthgd,phd->nthgp", q, kp)
    so = torch.einsum("nthgd,nphd->nthgp", q, ko).masked_fill(~seen[:, :, None, None], float("-inf"))
    top = so.amax(-1, keepdim=True)
    if c["prefix"]:
        top = torch.maximum(top, sp.amax(-1, keepdim=True))
    safe = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    sp, so = torch.exp(sp - safe), torch.exp(so - safe)
    total = sp.sum(-1) + so.sum(-1)
    o = torch.einsum("nthgp,phd->nthgd", sp, vp) + torch.einsum("nthgp,nphd->nthgd", so, vo)
    o = torch.where(total[..., None] > 0, o / total[..., None], torch.zeros_like(o))
    return o.reshape(s["q"].shape).to(s["q"].dtype), (torch.log(total) + safe[..., 0]).reshape(n, t, c["hq"])


def _weights(s, p, slots=None):
    """Matrices of projection p (0 gate, 1 up, 2 down) of the slots, [slots, rows, columns] in 32 bits."""
    c = s["case"]
    d, f, n = c["d"], c["f"], c["held"] + c["shared"]
    rows, cols = (d, f) if p == 2 else (f, d)
    w = s["arena"][:3 * n * d * f * SIZE[c["w"]]].view(TYPES[c["w"]] if c["w"] != "e4m3" else torch.uint8)
    if c["fused"]:
        w = w[2 * n * d * f:].view(n, rows, cols) if p == 2 else w[:2 * n * d * f].view(n, 2, rows, cols)[:, p]
    else:
        w = w.view(3, n, rows, cols)[p]
    w = w if slots is None else w[slots]
    if c["w"] != "e4m3":
        return w.float()
    rb, cb = -(-rows // 128), -(-cols // 128)
    scale = s["arena"][-3 * n * rb * cb * 4:].view(torch.float32).view(3, n, rb, cb)[p]
    scale = scale if slots is None else scale[slots]
    scale = scale.repeat_interleave(128, 1)[:, :rows].repeat_interleave(128, 2)[:, :, :cols]
    return w.view(torch.float8_e4m3fn).float() * scale


def _moe(s):
    c = s["case"]
    t, k, shared = c["tokens"], c["k"], c["shared"]
    logits, ids = s["logits"].sort(dim=-1, descending=True, stable=True)   # ties: the lowest index first
    p = torch.exp(logits - logits[:, :1])
    p = p[:, :k] / p[:, :k].sum(-1, keepdim=True)                           # softmax over all, renormalised over the chosen
    ids = ids[:, :k]
    every = torch.cat([ids, torch.arange(c["experts"], c["experts"] + shared, device="cuda").expand(t, -1)], 1)
    weight = torch.cat([p, torch.ones(t, shared, device="cuda")], 1)
    slots = s["slot_of_expert"].long()[every]
    weight = torch.where(slots >= 0, weight, torch.zeros_like(weight))
    x = s["x"].float()
    if slots.numel() < c["held"] + shared:   # few pairs: gather their matrices
        at = slots.clamp(min=0).reshape(-1)
        x = x.repeat_interleave(k + shared, 0)[:, :, None]
        g, u = _weights(s, 0, at) @ x, _weights(s, 1, at) @ x
        y = (_weights(s, 2, at) @ (g * torch.sigmoid(g) * u))[..., 0].view(t, k + shared, -1)
        out = (y * weight[..., None]).sum(1)
    else:                                    # every held expert on every token, then the weights
        dense = torch.zeros(t, c["held"] + shared, device="cuda").scatter_add_(1, slots.clamp(min=0), weight)
        g, u = x @ _weights(s, 0).transpose(1, 2), x @ _weights(s, 1).transpose(1, 2)
        h = g * torch.sigmoid(g) * u * dense.t()[:, :, None]
        out = torch.bmm(h, _weights(s, 2).transpose(1, 2)).sum(0)
    return out.to(s["x"].dtype), ids.int(), p


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    c = case
    if c["op"] in ("append", "gather"):
        per = c["hd"] * (SIZE[c["io"]] + SIZE[c["kv"]]) + (1 if c["kv"] == "e4m3" else 0)
        return {"bytes": c["tokens"] * (2 * c["heads"] * per + 8), "flops": 0}
    if c["op"] == "attend":
        lens = _lens(c)
        per = 2 * c["hkv"] * (c["hd"] * SIZE[c["kv"]] + (1 if c["kv"] == "e4m3" else 0))
        rows = c["qlen"] * c["hq"]
        pairs = sum(c["prefix"] + max(0, int(n) - c["qlen"] + i + 1) for n in lens for i in range(c["qlen"]))
        return {"bytes": (c["prefix"] + int(lens.sum())) * per + c["seqs"] * rows * (2 * c["hd"] * SIZE[c["io"]] + 4),
                "flops": 4 * c["hq"] * c["hd"] * pairs}
    m, used, pairs, tries = c["d"] * c["f"], 0, 0, 8
    host = np.random.RandomState(1)
    for _ in range(tries):   # expected number of experts in use
        top = np.argsort(-_logits(c, host), axis=1)[:, :c["k"]]
        held = host.permutation(c["experts"])[:c["held"]]
        hit = np.isin(top, held)
        used += len(np.unique(top[hit])) / tries
        pairs += hit.sum() / tries
    used, pairs = used + c["shared"], pairs + c["shared"] * c["tokens"]
    per = 3 * m * SIZE[c["w"]] + (3 * -(-c["d"] // 128) * -(-c["f"] // 128) * 4 if c["w"] == "e4m3" else 0)
    return {"bytes": used * per + c["tokens"] * (2 * c["d"] * SIZE[c["io"]] + 4 * c["experts"] + 8 * c["k"]), "flops": 6.0 * m * float(pairs)}


# ---- the definitions in 64 bits -----------------------------------------------------------------


def _exact_codes(x):
    """Codes as the values they are, and scales, of finite vectors along the last axis."""
    x = x.double()
    top = x.abs().amax(-1)
    k = torch.round(torch.log2(torch.where(top > 0, top, 448.0) / 448)) - 1   # at most the wanted one, two less at worst
    k = k + (448 * torch.exp2(k) < top).double()
    k = (k + (448 * torch.exp2(k) < top).double()).clamp(min=-126)
    k = torch.where(top > 0, k, 0.0)
    y = x / torch.exp2(k)[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -30))).clamp(min=-6) - 3)
    return torch.round(y / step) * step, torch.exp2(k)


def _exact_cache(s, i, block, off):
    """Vector(s) [heads, hd] of one token position, in 64 bits."""
    c = s["case"]
    x = (s["arena"][i, block, :, off] if c["hm"] else s["arena"][i, block, off])
    x = x.view(TYPES[c["kv"]]).double()
    if c["kv"] == "e4m3":
        scale = s["scales"][i, block, :, off] if c["hm"] else s["scales"][i, block, off]
        x = x * torch.exp2(scale.double() - 127)[..., None]
    return x


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "append":
        codes = s["arena"].view(TYPES[c["kv"]]).double()
        scales = torch.exp2(s["scales"].double() - 127) if c["kv"] == "e4m3" else None
        for i, x in enumerate((s["k"], s["v"])):
            v, sc = _exact_codes(x) if c["kv"] == "e4m3" else (x.double(), None)
            b, o = torch.div(s["slots"], c["block"], rounding_mode="floor"), s["slots"].remainder(c["block"])
            if c["hm"]:
                codes[i].transpose(1, 2)[b, o] = v
                if sc is not None:
                    scales[i].transpose(1, 2)[b, o] = sc
            else:
                codes[i][b, o] = v
                if sc is not None:
                    scales[i][b, o] = sc
        return (codes, scales) if c["kv"] == "e4m3" else codes
    if c["op"] == "gather":
        b, o = torch.div(s["slots"], c["block"], rounding_mode="floor"), s["slots"].remainder(c["block"])
        return _exact_cache(s, 0, b, o), _exact_cache(s, 1, b, o)
    if c["op"] == "attend":
        lens, table = s["lens"].tolist(), s["table"].long()
        group = c["hq"] // c["hkv"]
        q = s["q"].double()
        out, lse = torch.zeros_like(q), torch.full(q.shape[:3], float("-inf"), dtype=torch.float64, device="cuda")

        def read(blocks, count):
            pos = torch.arange(count, device="cuda")
            b, o = blocks[torch.div(pos, c["block"], rounding_mode="floor")], pos.remainder(c["block"])
            return _exact_cache(s, 0, b, o), _exact_cache(s, 1, b, o)

        pk, pv = read(s["prefix_table"].long(), c["prefix"])
        for h in range(c["hkv"]):
            ph, pw = pk[:, h].contiguous(), pv[:, h].contiguous()
            for i, n in enumerate(lens):
                k, v = read(table[i], n)
                k, v = torch.cat([ph, k[:, h]]), torch.cat([pw, v[:, h]])
                for t in range(c["qlen"]):
                    end = c["prefix"] + n - c["qlen"] + t + 1
                    if end <= 0:
                        continue
                    score = q[i, t, h * group:(h + 1) * group] @ k[:end].t() / math.sqrt(c["hd"])
                    lse[i, t, h * group:(h + 1) * group] = torch.logsumexp(score, -1)
                    out[i, t, h * group:(h + 1) * group] = torch.softmax(score, -1) @ v[:end]
        return out, lse
    logits = s["logits"].double().cpu().numpy()
    order = np.lexsort((np.broadcast_to(np.arange(c["experts"]), logits.shape), -logits), axis=-1)[:, :c["k"]]
    p = np.take_along_axis(logits, order, 1)
    p = np.exp(p - p.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    out = torch.zeros(c["tokens"], c["d"], dtype=torch.float64, device="cuda")
    slot = s["slot_of_expert"].tolist()
    n, d, f, size = c["held"] + c["shared"], c["d"], c["f"], SIZE[c["w"]]

    def matrix(j, proj):
        rows, cols = (d, f) if proj == 2 else (f, d)
        at = (2 * n + j if proj == 2 else 2 * j + proj) if c["fused"] else proj * n + j
        w = s["arena"][at * d * f * size:(at + 1) * d * f * size].view(TYPES[c["w"]]).double().view(rows, cols)
        if c["w"] == "e4m3":
            rb, cb = -(-rows // 128), -(-cols // 128)
            first = -(-3 * n * d * f // 256) * 256 + (proj * n + j) * rb * cb * 4
            scale = s["arena"][first:first + rb * cb * 4].view(torch.float32).double().view(rb, cb)
            w = w * scale[torch.arange(rows, device="cuda") // 128][:, torch.arange(cols, device="cuda") // 128]
        return w

    for e in range(c["experts"] + c["shared"]):
        if slot[e] < 0:
            continue
        if e < c["experts"]:
            t, where = np.nonzero(order == e)
            weight = torch.from_numpy(p[t, where]).cuda()
        else:
            t, weight = np.arange(c["tokens"]), torch.ones(c["tokens"], dtype=torch.float64, device="cuda")
        if not len(t):
            continue
        x = s["x"][torch.from_numpy(t).cuda()].double()
        g = x @ matrix(slot[e], 0).t()
        h = g / (1 + torch.exp(-g)) * (x @ matrix(slot[e], 1).t())
        out.index_add_(0, torch.from_numpy(t).cuda(), weight[:, None] * (h @ matrix(slot[e], 2).t()))
    return out, torch.from_numpy(order.astype(np.int32)), torch.from_numpy(p)


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(4)]:
        print(c, work(c))
