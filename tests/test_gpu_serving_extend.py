"""emoe_kv_extend and emoe_kv_keep on the GPU against their definitions: whole numbers and copies, equal to the last bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import rows_ref as RR
import serving_ref as R
from test_gpu_serving_kv import device_cache, filled, same

pytestmark = pytest.mark.gpu


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


def handle(pool, block, status=None):
    return E.KvCache(1 << 20, n_layers=1, num_blocks=pool, block_tokens=block, n_heads=1, head_dim=8, status=status)


def run(lens, add, table, free, n_free, n_slots, block, pool, in_place=False, graph=False):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = handle(pool, block, status)
    t = [dev(lens), dev(add), dev(table), dev(free), dev([n_free]), dev(np.full(len(lens) + 1, -7)), dev(np.full(n_slots, -7), np.int64),
         dev(np.full(len(lens), -7)), dev([-7])]
    if in_place:
        t[7], t[8] = t[0], t[4]
    c.extend(*t)
    torch.cuda.synchronize()
    names = ("lens_out", "table", "free", "n_free", "q_start", "slots", "status")
    got = [x.cpu().numpy().tolist() for x in (t[7], t[2], t[3], t[8], t[5], t[6], status)]
    return dict(zip(names, got))


def check(lens, add, table, free, n_free, n_slots, block, pool, **kw):
    got = run(lens, add, table, free, n_free, n_slots, block, pool, **kw)
    want = RR.extend(lens, add, table, free, n_free, n_slots, block, pool)
    for name, w in zip(("lens_out", "table", "free", "n_free", "q_start", "slots", "status"), want):
        g = got[name]
        if name in ("n_free", "status"):
            w = [w]
        elif name in ("table",):
            w = [list(map(int, r)) for r in w]
        else:
            w = list(map(int, w))
        if name == "status" and set(g + w) <= {4, 11}:
            continue   # two things to report: one of them is
        assert g == w, name
    return got


def batch(seed, n, block, top, add_hi, back, spare, short=0):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, top + 1, n)
    add = rng.integers(0, add_hi + 1, n)
    gone = rng.random(n) < back
    add[gone] = -rng.integers(0, top + 5, gone.sum())
    width = -(-(top + add_hi) // block)
    held = [-(-int(x) // block) for x in lens]
    pool = sum(held) + spare
    ids = rng.permutation(pool)
    table = np.full((n, max(1, width)), -1)
    at = 0
    for i, m in enumerate(held):
        table[i, :m] = ids[at:at + m]
        at += m
    free = np.full(pool + 3, -1)
    free[:spare] = ids[at:]
    return lens.tolist(), add.tolist(), table.tolist(), free.tolist(), spare, int(np.maximum(add, 0).sum()) + 3 - short, block, pool


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,block,top,add_hi,back,spare", [
    (1, 16, 0, 1, 0, 1), (1, 16, 100, 5000, 0, 400), (64, 16, 2750, 1, 0, 100), (33, 1, 20, 7, 0.3, 300), (1000, 16, 300, 127, 0.2, 9000),
    (1025, 7, 50, 9, 0.5, 2000), (8192, 8, 40, 3, 0.3, 9000), (3, 64, 9000, 30000, 0, 2000), (40, 16, 100, 0, 1, 0), (31, 24, 70, 40, 0.4, 60)])
def test_extend(n, block, top, add_hi, back, spare, in_place):
    check(*batch(n + block, n, block, top, add_hi, back, spare), in_place=in_place)


@pytest.mark.parametrize("n", [5, 77, 1500])
def test_extend_when_blocks_run_out(n):
    """Too few blocks, too few slots, rows that are too short: each sequence is served or refused as a whole."""
    a = list(batch(n, n, 8, 60, 30, 0.2, n // 2))
    check(*a)
    a = list(batch(n + 1, n, 8, 60, 30, 0.1, 10 * n, short=n * 4))
    check(*a)
    lens, add, table, free, n_free, n_slots, block, pool = batch(n + 2, n, 8, 60, 30, 0.1, 10 * n)
    check(lens, add, [r[:8] for r in table], free, n_free, n_slots, block, pool)      # rows of 64 tokens
    check(lens, add, table, free[:n_free + 2], n_free, n_slots, block, pool)            # no room for what is given back
    check(lens, add, table, free, 0, n_slots, block, pool)


def test_extend_at_its_limits():
    table = [[5, 6], [7, 8]]
    check([0, 0], [0, 0], table, [1, 2], 2, 0, 4, 9)                   # nothing to do, no slot map
    check([-3, 8], [4, -100], table, [1, 2, 0, 0], 2, 4, 4, 9)         # a length below zero, all tokens gone and more
    check([8, 8], [1, -1], table, [1, 2], 2, 4, 4, 9)                  # a row that is full already
    check([20, 8], [-1, -9], table, [1, 2, 0, 0, 0], 2, 4, 4, 9)       # a length beyond the row
    check([3, 3], [2 ** 31 - 1, 1], table, [1, 2], 2, 4, 4, 9)         # more than any row
    check([2 ** 31 - 1, 3], [2 ** 31 - 1, 1], table, [1, 2], 2, 4, 4, 9)
    check([3, 3], [2, -2 ** 31], table, [1, 2, 0], 2, 4, 4, 9)
    check([3, 4], [2, 1], table, [1, 99], 2, 4, 4, 9)                  # an id outside the pool in the list
    check([3, 4], [1, -4], [[-1, -1], [-2, 3]], [1, 2, 0], 2, 4, 4, 9)  # and in the table
    check([3, 4], [1, -4], table, [1, 2, 0], 1 << 30, 4, 4, 9)         # more free blocks than the list has
    check([3, 4], [1, 1], table, [1, 2, 0], -1, 4, 4, 9)


def test_extend_an_empty_batch():
    c = handle(9, 4)
    q_start, slots, left = dev([5]), dev([5, 5, 5], np.int64), dev([5])
    c.extend(dev([]), dev([]), dev(np.zeros((0, 3))), dev([1, 2]), dev([2]), q_start, slots, dev([]), left)
    assert q_start.tolist() == [0] and slots.tolist() == [-1] * 3 and left.tolist() == [2]


def test_extend_captured_follows_the_lengths():
    """A step of one token a sequence, captured once: tables, lengths and the list go on from replay to replay."""
    block, pool = 4, 40
    table, free, lens = np.full((3, 12), -1), list(range(pool)), [0, 3, 9]
    ids = iter(range(pool - 1, -1, -1))
    for s, n in enumerate(lens):
        for j in range(-(-n // block)):
            table[s, j] = next(ids)
    n_free = pool - sum(-(-n // block) for n in lens)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = handle(pool, block, status)
    d = dict(lens=dev(lens), add=dev([1, 1, 1]), block_table=dev(table), free_blocks=dev(free), n_free=dev([n_free]), q_start=dev([0] * 4),
             slots=dev([0] * 5, np.int64))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.extend(**d, lens_out=d["lens"], n_free_out=d["n_free"], stream=torch.cuda.current_stream())
    state = (lens, table.tolist(), free, n_free)
    for _ in range(15):
        graph.replay()
        out, tab, fr, left, start, slots, st = RR.extend(state[0], [1, 1, 1], state[1], state[2], state[3], 5, block, pool)
        state = (out, tab, fr, left)
        assert d["lens"].tolist() == out and d["block_table"].tolist() == tab and d["free_blocks"].tolist() == fr and d["n_free"].tolist() == [left]
        assert d["q_start"].tolist() == start and d["slots"].tolist() == slots and status.item() == st == 0


KEEPS = [
    # block, KV heads, hd, cache, head major, layers, lengths, nodes, most
    (16, 4, 128, "bf16", False, 2, [100, 30, 26], [26, 26, 26], 6), (16, 1, 128, "e4m3", True, 3, [70, 64], [64, 1], 9), (5, 3, 72, "f16", True, 1, [9, 40], [9, 13], 4),
    (1, 2, 8, "e4m3", False, 2, [50], [40], 20), (8, 5, 24, "e4m3", True, 1, [33, 12, 0], [20, 12, 0], 12), (16, 2, 256, "bf16", False, 5, [400], [300], 64),
    (32, 16, 64, "f16", False, 1, [90] * 20, [13] * 20, 3),
]


@pytest.mark.parametrize("block,hkv,hd,kv,hm,layers,lens,nodes,most", KEEPS)
def test_keep(block, hkv, hd, kv, hm, layers, lens, nodes, most):
    rng = np.random.default_rng(block + hd)
    held = [-(-n // block) for n in lens]
    pool = sum(held) + 2
    ref = filled(rng, (layers, pool, block, hkv), hd, kv, hm)
    ids, table = list(rng.permutation(pool)), np.full((len(lens), max(held) + 1), -1)
    for i, m in enumerate(held):
        table[i, :m] = [ids.pop() for _ in range(m)]
    accepted, count = np.full((len(lens), most), -1), []
    for i, n in enumerate(nodes):
        m = int(rng.integers(0, min(n, most) + 1))
        accepted[i, :m] = np.sort(rng.permutation(n)[:m])   # dense paths overlap their new places
        count.append(m)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, arena, scales = device_cache(ref, status=status)
    starts = np.concatenate([[0], np.cumsum(nodes)])
    change = dev([-99] * len(lens))
    c.keep(dev(table), dev(lens), dev(starts), dev(accepted), dev(count), change)
    moves, want = RR.keep(lens, starts, accepted, count, most)
    before = ref.values.copy(), ref.bytes.copy()
    for s, a, b in moves:
        at, to = (table[s, a // block], a % block), (table[s, b // block], b % block)
        ref.values[:, :, to[0], to[1]], ref.bytes[:, :, to[0], to[1]] = before[0][:, :, at[0], at[1]], before[1][:, :, at[0], at[1]]
    assert change.tolist() == want and status.item() == 0
    same(arena, scales, ref)


@pytest.mark.parametrize("path,count,moved,word", [
    ([1, 1, 3], 3, 1, 4), ([3, 2, 4], 3, 1, 4), ([0, 8, 2], 3, 1, 4), ([-1, 2, 3], 3, 0, 4), ([1, 3, 5], -2, 0, 0), ([1, 3, 5], 9, 3, 4), ([2, 3, 7], 2, 2, 0)])
def test_keep_of_paths_that_do_not_rise(path, count, moved, word):
    ref = filled(np.random.default_rng(4), (1, 5, 8, 2), 64, "bf16", False)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, arena, _ = device_cache(ref, status=status)
    change = dev([0])
    c.keep(dev([[3, 1, 4]]), dev([20]), dev([0, 8]), dev([path]), dev([count]), change)
    flat = ref.values[0].reshape(2, 40, 2, 64).copy()
    slot = lambda p: [3, 1, 4][p // 8] * 8 + p % 8    # noqa: E731
    for i in range(moved):
        ref.values[0].reshape(2, 40, 2, 64)[:, slot(12 + i)] = flat[:, slot(12 + path[i])]
    assert change.tolist() == [moved - 8] and status.item() == word
    same(arena, None, ref)


def test_keep_with_places_that_are_not_there():
    """A block outside the pool, a place beyond the table, more nodes than tokens: left out and reported."""
    for table, lens, nodes in (([[3, 77, 4]], 20, 8), ([[3, 1]], 20, 8), ([[3, -1, 4]], 20, 8), ([[3, 1, 4]], 2, 8)):
        ref = filled(np.random.default_rng(4), (1, 5, 8, 2), 64, "bf16", False)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        c, arena, _ = device_cache(ref, status=status)
        change = dev([0])
        c.keep(dev(table), dev([lens]), dev([0, nodes]), dev([[2, 5, 7]]), dev([3]), change)
        flat = ref.values[0].reshape(2, 40, 2, 64).copy()

        def slot(p):
            b = table[0][p // 8] if 0 <= p < 8 * len(table[0]) else -1
            return b * 8 + p % 8 if 0 <= b < 5 else -1
        for i, x in enumerate((2, 5, 7)):
            a, b = slot(lens - nodes + x), slot(lens - nodes + i)
            if a >= 0 and b >= 0:
                ref.values[0].reshape(2, 40, 2, 64)[:, b] = flat[:, a]
        assert change.tolist() == [-5] and status.item() == 4
        same(arena, None, ref)


def test_drafting_step_by_step():
    """Extend, append, attend_tree, keep, extend: two steps of drafting leave the cache that appending the accepted tokens alone leaves."""
    rng = np.random.default_rng(9)
    block, hkv, hd, pool, n = 8, 2, 64, 60, 3
    ref = R.Cache(2, pool, block, hkv, hd, "bf16")
    c, arena, _ = device_cache(ref)
    lens, q_start, change, n_free = dev([5, 16, 0]), dev([0] * (n + 1)), dev([0] * n), dev([pool])
    table, free, slots = dev(np.full((n, 10), -1)), dev(np.arange(pool)), dev(np.zeros(64), np.int64)
    start = lens.clone()
    lens.zero_()
    step = lambda add: c.extend(lens, add, table, free, n_free, q_start, slots, lens, n_free)    # noqa: E731
    step(start)
    kept = [[], [], []]
    x = torch.from_numpy(rng.standard_normal((2, 64, 2, hkv, hd))).to(torch.bfloat16).cuda()

    def append():
        for layer in range(2):
            c.append(layer, x[layer, :, 0], x[layer, :, 1], slots)
    append()
    at = q_start.tolist()
    for s in range(n):
        kept[s] += [x[:, i].clone() for i in range(at[s], at[s + 1])]
    for nodes, paths in (([7, 5, 9], [[0, 2, 5], [0], [0, 1, 2, 8]]), ([6, 1, 12], [[], [0], [0, 3, 4]])):
        x = torch.from_numpy(rng.standard_normal((2, 64, 2, hkv, hd))).to(torch.bfloat16).cuda()
        step(dev(nodes))
        append()
        at = q_start.tolist()
        q = torch.from_numpy(rng.standard_normal((64, 4, hd))).to(torch.bfloat16).cuda()
        out, mask = torch.empty_like(q), torch.full((64, 1), -1, dtype=torch.int32, device="cuda")
        work = torch.empty(max(1, c.attend_tree_workspace_bytes(n, 64, 12, 4, 10)), dtype=torch.uint8, device="cuda")
        c.attend_tree(1, q, out, table, lens, q_start, mask, 12, workspace=work)
        for s in range(n):
            seq = torch.stack(kept[s] + [x[:, i] for i in range(at[s], at[s + 1])], 1)[1].double()    # [tokens, K or V, heads, hd]
            for h in range(4):
                p = torch.softmax(q[at[s]:at[s + 1], h].double() @ seq[:, 0, h // 2].T * hd ** -0.5, -1)
                want, a = p @ seq[:, 1, h // 2], p @ seq[:, 1, h // 2].abs()
                assert ((out[at[s]:at[s + 1], h].double() - want).abs() <= 2.2 * 2.0 ** -8 * a).all()
        accepted = np.full((n, 4), -1)
        for s, p in enumerate(paths):
            accepted[s, :len(p)] = p
            kept[s] += [x[:, at[s] + i].clone() for i in p]
        c.keep(table, lens, q_start, dev(accepted), dev([len(p) for p in paths]), change)
        step(change)
    assert lens.tolist() == [len(k) for k in kept]
    assert n_free.item() == pool - sum(-(-len(k) // block) for k in kept)
    view, tab = arena.view(torch.bfloat16).view(2, 2, pool, block, hkv, hd), table.tolist()
    for s in range(n):
        for j, want in enumerate(kept[s]):
            assert torch.equal(view[:, :, tab[s][j // block], j % block], want)
