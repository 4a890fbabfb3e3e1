"""Plain 64-bit definitions of the operators on packed query tokens: masks as truth values, attention over them on
torch tensors, block tables and paths with python lists.  Test infrastructure."""
from __future__ import annotations

import numpy as np
import torch

import serving_ref as R


def window_sees(length, count, window, sinks):
    """[count, length]: which tokens each of the last `count` tokens sees."""
    place, j = length - count + np.arange(count)[:, None], np.arange(length)[None]
    return (j <= place) & ((j > place - window) | (j < sinks))


def tree_sees(length, count, bits):
    """bits [count, count] of truth values (row: node, column: node that it sees)."""
    sees = np.ones((count, max(length, count)), bool)
    sees[:, sees.shape[1] - count:] = bits
    return sees[:, sees.shape[1] - length:]


def packed_bits(rows, words):
    """Truth values [n, up to 32 * words] -> int32 [n, words]."""
    out = np.zeros((len(rows), words * 32), bool)
    out[:, :rows.shape[1]] = rows
    return np.packbits(out.reshape(len(rows), words, 4, 8), axis=-1, bitorder="little")[..., 0].reshape(len(rows), words * 4).view("<i4")


def attend(ref, layer, q, table, lens, starts, sees, scale):
    """q [tokens, Hq, hd] float64 on any device; sees[s]: [count, length].  Returns out, lse, a = sum p |v| and e, the bound of a
    score's error (as in serving_ref.attend), and for an e4m3 cache f: its weights are f16 with a step of 2^-30 of the largest
weight times the largest scale of v that the row sees, half of which each of its codes may be off by.  What a row does not
see has no part in any of them."""
    heads, block, dev = ref.dims[4], ref.dims[3], q.device
    group, hd = q.shape[1] // heads, q.shape[2]
    o, a = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], float("-inf"), dtype=torch.float64, device=dev)
    err, far = torch.zeros_like(lse), torch.zeros_like(q)
    values = ref.values[layer] * (R.scale_value(ref.bytes[layer])[..., None] if ref.kv_type == "e4m3" else 1.0)
    for s in range(len(lens)):
        first, count = starts[s], starts[s + 1] - starts[s]
        if count == 0 or lens[s] == 0:
            continue
        j = np.arange(lens[s])
        ids = table[s][j // block]
        inside = (ids >= 0) & (ids < ref.dims[2])
        see = torch.from_numpy(sees[s] & inside[None]).to(dev)
        kv = torch.from_numpy(values[:, np.where(inside, ids, 0), j % block]).to(dev)
        for h in range(q.shape[1]):
            k, v = kv[0, :, h // group], kv[1, :, h // group]
            x = q[first:first + count, h]
            score = (scale * (x @ k.T)).masked_fill(~see, float("-inf"))
            # each row's products are made of what it sees alone: 0 * NaN of a token beside them would be NaN
            top = torch.where(see, score, float("-inf")).amax(-1, keepdim=True)
            safe = torch.where(torch.isinf(top) & (top < 0), 0.0, top)
            w = torch.where(see, torch.exp(score - safe), 0.0)
            total = w.sum(-1, keepdim=True)
            some = see.any(-1)
            odd = ~torch.isfinite(v).all(-1)
            part = w @ torch.where(odd[:, None], 0.0, v)
            for t in torch.nonzero(odd).flatten().tolist():
                part = part + torch.where(see[:, t, None], w[:, t, None] * v[t], 0.0)
            o[first:first + count, h] = torch.where(some[:, None], part / torch.where(total == 0, 1.0, total), 0.0)
            a[first:first + count, h] = torch.where(some[:, None], (w @ v.abs().nan_to_num(0, 0, 0)) / torch.where(total == 0, 1.0, total), 0.0)
            lse[first:first + count, h] = torch.where(some, (safe + torch.log(total))[:, 0], float("-inf"))
            size = abs(scale) * torch.where(see, x.abs() @ k.abs().T, 0.0).nan_to_num(0, 0, 0).amax(-1)
            err[first:first + count, h] = (hd + 8) * 2.0 ** -23 * size + (lens[s] + 16) * 2.0 ** -23
            if ref.kv_type == "e4m3":
                codes = torch.from_numpy(np.abs(ref.values[layer, 1][np.where(inside, ids, 0), j % block, h // group])).to(dev).nan_to_num(0)
                byte = torch.from_numpy(ref.bytes[layer, 1][np.where(inside, ids, 0), j % block, h // group].astype(np.float64)).to(dev)
                most = torch.where(see & (byte < 255), torch.exp2(byte - 127), 0.0).amax(-1, keepdim=True)
                far[first:first + count, h] = 2.0 ** -31 * most * (see.double() @ codes) / torch.where(total == 0, 1.0, total).nan_to_num(1)
    return o, lse, a, err, far


def extend(lens, add, table, free, n_free, n_slots, block, pool):
    """Everything that emoe_kv_extend writes, and the status: (lens_out, table, free, n_free_out, q_start, slots, status)."""
    table, free, status = [list(r) for r in table], list(free), 0
    n, width, room = len(lens), len(table[0]) if len(table) else 0, len(free)
    lens, top = [max(0, int(x)) for x in lens], min(max(0, n_free), room)
    blocks = lambda x: -(-x // block)    # noqa: E731
    out, start, total, wanted = list(lens), [], 0, 0
    for s in range(n):   # what is given back
        if add[s] < 0:
            out[s] = max(0, lens[s] + int(add[s]))
            for col in range(blocks(out[s]), min(width, blocks(lens[s]))):
                if top < room:
                    free[top] = table[s][col]
                    top += 1
                else:
                    status = 11
                if not 0 <= table[s][col] < pool:
                    status = status or 4
    granted, taken = [], 0
    for s in range(n):
        m = max(0, int(add[s]))
        start.append(min(total, n_slots))
        total += m
        fits = m == 0 or blocks(lens[s] + m) <= width
        need = blocks(lens[s] + m) - min(width, blocks(lens[s])) if m and fits else 0
        wanted += need
        granted.append(fits and (m == 0 or total <= n_slots) and (need == 0 or wanted <= top))
        if not granted[s]:
            status = 11
        elif m:
            out[s] = lens[s] + m
            for col in range(blocks(lens[s]), blocks(out[s])):
                table[s][col] = free[top - 1 - taken]
                taken += 1
    start.append(min(total, n_slots))
    slots = [-1] * n_slots
    for s in range(n):
        if granted[s]:
            for i in range(max(0, int(add[s]))):
                p = lens[s] + i
                if 0 <= table[s][p // block] < pool:
                    slots[start[s] + i] = table[s][p // block] * block + p % block
                else:
                    status = status or 4
    return out, table, free, top - taken, start, slots, status


def keep(lens, starts, accepted, n_accepted, most):
    """[(sequence, from place, to place)] in order, and the change of each sequence."""
    moves, change = [], []
    for s in range(len(lens)):
        nodes, count = starts[s + 1] - starts[s], 0
        for i in range(min(max(0, n_accepted[s]), most)):
            x = accepted[s][i]
            if not 0 <= x < nodes or (i and x <= accepted[s][i - 1]):
                break
            moves.append((s, lens[s] - nodes + x, lens[s] - nodes + i))
            count += 1
        change.append(count - nodes)
    return moves, change
