"""The serving operators together with the re-layout: decode steps on the old ranks' arenas, the scale
step, the same decode steps on the new ranks' - append, attend and the expert layer, 16-bit and
quantised - against the 64-bit definitions on the logical state, which the step does not change."""
from __future__ import annotations

import dataclasses

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import serving_ref as R
import workloads as W
from test_gpu_serving_attend import HALF_STEP
from test_gpu_serving_kv import TORCH

pytestmark = pytest.mark.gpu

D, F, HQ, HKV, HD, BLOCK = 256, 96, 8, 4, 64, 16
LAYERS, EXPERTS, SHARED, TOP_K = 2, 9, 1, 3
PREFIX, LENS, GROW = 37, [20, 5, 33], 3      # tokens before the step; GROW more after it


def configs():
    """EP2 -> EP3 with a replicated expert, TP2 -> TP4, a new block table."""
    rng = np.random.default_rng(0)
    total = [PREFIX] + [n + 2 * GROW for n in LENS]      # the prefix is a sequence of its own in the tables
    blocks = [-(-n // BLOCK) for n in total]
    out = []
    for ep, tp, pool, placement in ((2, 2, sum(blocks) + 2, [[0, 2, 4, 6, 8, 9], [1, 3, 5, 7, 9]]),
                                    (3, 4, sum(blocks) + 5, [[0, 3, 6, 9], [1, 4, 7, 8, 9], [2, 5, 8, 9]])):
        ids = list(rng.permutation(pool))
        table = np.full((len(total), max(blocks)), -1, np.int32)
        for i, n in enumerate(blocks):
            table[i, :n] = [ids.pop() for _ in range(n)]
        out.append(W.ParallelConfig(ep, tp, placement, pool, total, table))
    return out


class Ranks:
    """One side's arenas and handles: KV caches by TP rank, expert arenas by EP rank."""

    def __init__(self, cfg, kv_type, w_type, shape, plans, side):
        self.cfg = cfg
        zeros = lambda plan, ph: [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in plan.arena_bytes(ph, side)]   # noqa: E731
        self.kv = zeros(plans["kv"], E.PHASE_KV)
        self.scales = zeros(plans["scales"], E.PHASE_KV) if kv_type == "e4m3" else [None] * cfg.tp
        self.experts = zeros(plans["experts"], E.PHASE_EXPERTS)
        kv_shape = dataclasses.replace(shape, elem_bytes=R.TYPE_BYTES[kv_type])
        self.caches = [E.KvCache.for_rank(kv_shape, cfg.tp, cfg.kv_num_blocks, a, kv_type, scales=s) for a, s in zip(self.kv, self.scales)]
        self.layers = [E.ExpertArena.for_rank(dataclasses.replace(shape, elem_bytes=R.TYPE_BYTES[w_type]), len(p), a, w_type)
                       for p, a in zip(cfg.placement, self.experts)]
        self.table = torch.from_numpy(cfg.block_table).cuda()
        self.slots = []          # per rank: slot of each expert that this rank's call takes; replicas go to the first rank
        taken = set()
        for p in cfg.placement:
            t = [-1] * (EXPERTS + SHARED)
            for s, e in enumerate(p):
                if e not in taken:
                    t[e] = s
                    taken.add(e)
            self.slots.append(torch.tensor(t, dtype=torch.int32, device="cuda"))

    def token_slots(self, seq, first, n):
        at = torch.arange(first, first + n, device="cuda")
        return self.table[seq, at // BLOCK].long() * BLOCK + at % BLOCK

    def append(self, layer, k, v, slots):
        for t, c in enumerate(self.caches):
            mine = slice(t * HKV // self.cfg.tp, (t + 1) * HKV // self.cfg.tp)
            c.append(layer, k[:, mine], v[:, mine], slots)

    def attend(self, layer, q, lens):
        out = torch.empty_like(q)
        table = self.table[1:].contiguous()
        for t, c in enumerate(self.caches):
            mine = slice(t * HQ // self.cfg.tp, (t + 1) * HQ // self.cfg.tp)
            n = c.attend_workspace_bytes(len(LENS), 1, HQ // self.cfg.tp, table.shape[1], PREFIX)
            c.attend(layer, q[:, :, mine], out[:, :, mine], table, lens, self.table[0].contiguous(), PREFIX,
                     workspace=torch.empty(max(n, 1), dtype=torch.uint8, device="cuda"))
        return out

    def moe(self, layer, x, logits):
        total = torch.zeros(x.shape, device="cuda")
        for h, slots in zip(self.layers, self.slots):
            part = torch.empty(x.shape, device="cuda")
            work = torch.empty(h.decode_workspace_bytes(len(x), TOP_K, EXPERTS, SHARED), dtype=torch.uint8, device="cuda")
            h.decode(layer, x, logits, TOP_K, slots, part, n_shared=SHARED, workspace=work)
            total += part
        return total


@pytest.mark.parametrize("kv_type,w_type", [("bf16", "bf16"), ("e4m3", "e4m3")])
def test_decode_steps_around_a_scale_step(kv_type, w_type):
    rng = np.random.default_rng(1)
    old_cfg, new_cfg = configs()
    scale_bytes = (-(-D // 128)) * (-(-F // 128)) * 4 if w_type == "e4m3" else 0
    shape = W.Shape(LAYERS, EXPERTS, SHARED, D, F, HQ, HKV, HD, BLOCK, 2)
    sized = lambda **kw: dataclasses.replace(shape, **kw)    # noqa: E731
    plans = {"kv": E.Plan(sized(elem_bytes=R.TYPE_BYTES[kv_type]), old_cfg, new_cfg),
             "experts": E.Plan(sized(elem_bytes=R.TYPE_BYTES[w_type], expert_scale_bytes=scale_bytes), old_cfg, new_cfg)}
    if kv_type == "e4m3":
        plans["scales"] = E.Plan(sized(head_dim=1, elem_bytes=1), old_cfg, new_cfg)
    old, new = (Ranks(cfg, kv_type, w_type, shape, plans, side) for cfg, side in ((old_cfg, E.SIDE_OLD), (new_cfg, E.SIDE_NEW)))

    # expert matrices, logical and on the old ranks
    logical = {}
    for r, p in enumerate(old_cfg.placement):
        n, m = len(p), D * F
        for layer in range(LAYERS):
            for proj in range(3):
                for s, e in enumerate(p):
                    if (layer, proj, e) not in logical:
                        if w_type == "e4m3":
                            codes = torch.from_numpy(np.clip(rng.standard_normal(m) * 100, -440, 440)).float().to(torch.float8_e4m3fn)
                            scales = torch.from_numpy(rng.uniform(0.5, 1.5, scale_bytes // 4) / 100 / np.sqrt(D)).float()
                            logical[layer, proj, e] = (codes.view(torch.uint8), scales)
                        else:
                            logical[layer, proj, e] = (torch.from_numpy(rng.standard_normal(m) / np.sqrt(D)).to(torch.bfloat16).view(torch.uint8), None)
                    raw, sc = logical[layer, proj, e]
                    at = ((layer * 3 + proj) * n + s) * raw.numel()
                    old.experts[r][at:at + raw.numel()] = raw.cuda()
                    if sc is not None:
                        first = -(-3 * LAYERS * n * m // 256) * 256 + ((layer * 3 + proj) * n + s) * scale_bytes
                        old.experts[r][first:first + scale_bytes] = sc.view(torch.uint8).cuda()

    def matrix(layer, proj, e):
        rows, cols = (D, F) if proj == 2 else (F, D)
        raw, sc = logical[layer, proj, e]
        v = raw.view(TORCH[w_type]).double().numpy().reshape(rows, cols)
        if sc is not None:
            s = sc.double().numpy().reshape(-(-rows // 128), -(-cols // 128))
            v = v * s[np.arange(rows) // 128][:, np.arange(cols) // 128]
        return v

    # the logical cache: one sequence after the other, prefix first
    tokens = [PREFIX] + [n + 2 * GROW for n in LENS]
    kv = torch.from_numpy(rng.standard_normal((LAYERS, 2, sum(tokens), HKV, HD))).to(torch.bfloat16)
    starts = np.concatenate([[0], np.cumsum(tokens)])

    def held(layer, i, seq, n):
        x = kv[layer, i, starts[seq]:starts[seq] + n].double().numpy()
        if kv_type != "e4m3":
            return x
        codes, byte = R.quantise(x)
        return codes * R.scale_value(byte)[..., None]

    def decode_step(ranks, lens):
        """Appends a token to every sequence, attends, runs the experts; all against the definitions."""
        for layer in range(LAYERS):
            rows = [int(starts[s + 1] + n) for s, n in enumerate(lens)]
            slots = torch.cat([ranks.token_slots(s + 1, n, 1) for s, n in enumerate(lens)])
            fresh = kv[layer][:, rows].cuda()
            ranks.append(layer, fresh[0], fresh[1], slots)
            q = torch.from_numpy(rng.standard_normal((len(LENS), 1, HQ, HD)) * 2).to(torch.bfloat16).cuda()
            now = torch.tensor([n + 1 for n in lens], dtype=torch.int32, device="cuda")
            got = ranks.attend(layer, q, now).double().cpu().numpy()
            for s, n in enumerate(lens):
                k, v = (np.concatenate([held(layer, i, 0, PREFIX), held(layer, i, s + 1, n + 1)]) for i in range(2))
                for h in range(HQ):
                    qs = q[s, 0, h].double().cpu().numpy()
                    score = HD ** -0.5 * (k[:, h // 2] @ qs)
                    w = np.exp(score - score.max())
                    w /= w.sum()
                    a = w @ np.abs(v[:, h // 2])
                    e = (HD + 8) * 2.0 ** -23 * HD ** -0.5 * (np.abs(k[:, h // 2]) @ np.abs(qs)).max() + (len(k) + 16) * 2.0 ** -23
                    assert (np.abs(got[s, 0, h] - w @ v[:, h // 2]) <= 1.05 * (2 * HALF_STEP["bf16"] + 2 * e) * a).all()
            x = torch.from_numpy(rng.standard_normal((len(LENS), D))).to(torch.bfloat16).cuda()
            logits = torch.from_numpy(rng.standard_normal((len(LENS), EXPERTS))).float().cuda()
            got = ranks.moe(layer, x, logits).double().cpu().numpy()
            ids, p = R.route(logits.cpu().numpy(), TOP_K)
            p /= p.sum(1, keepdims=True)
            for t in range(len(LENS)):
                y, tol = np.zeros(D), np.zeros(D)
                xt = x[t].double().cpu().numpy()
                for e, w in list(zip(ids[t], p[t])) + [(EXPERTS, 1.0)]:
                    g, u = matrix(layer, 0, e) @ xt, matrix(layer, 1, e) @ xt
                    err = (D + 8) * 2.0 ** -23
                    dg, du = err * (np.abs(matrix(layer, 0, e)) @ np.abs(xt)), err * (np.abs(matrix(layer, 1, e)) @ np.abs(xt))
                    silu = g / (1 + np.exp(-g))
                    h = w * silu * u
                    y += matrix(layer, 2, e) @ h
                    # hidden values rounded once to bf16 (a step here: their weight is off by 1e-5 too), sums of 32 bits
                    tol += np.abs(matrix(layer, 2, e)) @ (abs(w) * (1.1 * np.abs(u) * dg + np.abs(silu) * du) + (2.0 ** -8 + 2e-5 + 4 * F * 2.0 ** -23) * np.abs(h))
                assert (np.abs(got[t] - y) <= 1.05 * tol + 1e-30).all()
        return [n + 1 for n in lens]

    for layer in range(LAYERS):   # the prompts
        for seq, n in [(0, PREFIX)] + [(s + 1, n) for s, n in enumerate(LENS)]:
            x = kv[layer][:, starts[seq]:starts[seq] + n].cuda()
            old.append(layer, x[0], x[1], old.token_slots(seq, 0, n))
    lens = list(LENS)
    for _ in range(GROW):
        lens = decode_step(old, lens)
    # the scale step: codes and scales under the same tables
    plans["kv"].reshard_kv(old.kv, new.kv)
    if kv_type == "e4m3":
        plans["scales"].reshard_kv(old.scales, new.scales)
    plans["experts"].reshard_experts(old.experts, new.experts)
    # what the new ranks hold is what the old ones held, bit for bit
    for layer in range(LAYERS):
        for seq, n in [(0, PREFIX)] + [(s + 1, n) for s, n in enumerate(lens)]:
            both = []
            for ranks in (old, new):
                parts = []
                for c in ranks.caches:
                    k, v = (torch.empty(n, c.n_heads, HD, dtype=torch.bfloat16, device="cuda") for _ in range(2))
                    c.gather(layer, ranks.token_slots(seq, 0, n), k, v)
                    parts.append(torch.stack([k, v]))
                both.append(torch.cat(parts, 2))
            assert torch.equal(both[0], both[1])
            assert np.array_equal(both[0][1].double().cpu().numpy(), held(layer, 1, seq, n))
    for _ in range(GROW):
        lens = decode_step(new, lens)
    for p in plans.values():
        p.close()
