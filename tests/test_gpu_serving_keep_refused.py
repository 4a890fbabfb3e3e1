"""Drafting when blocks run out: a sequence that emoe_kv_extend refuses has no nodes, and emoe_kv_keep, told by the slots, leaves
its tokens alone."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import serving_ref as R
from test_gpu_serving_extend import dev
from test_gpu_serving_kv import device_cache, filled, same

pytestmark = pytest.mark.gpu


def test_a_refused_sequence_keeps_its_tokens():
    """Blocks for the first of three trees only."""
    rng = np.random.default_rng(7)
    block, hkv, hd, pool, n = 4, 2, 64, 12, 3
    ref = filled(rng, (2, pool, block, hkv), hd, "bf16", False)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, arena, _ = device_cache(ref, status=status)
    table = dev([[4, 7] + [-1] * 4, [0, 9, 2] + [-1] * 3, [5] + [-1] * 5])
    lens, q_start, slots, change = dev([6, 11, 4]), dev([0] * 4), dev([0] * 20, np.int64), dev([-99] * 3)
    free, n_free = dev([1, 3, 6, 0, 0]), dev([2])
    c.extend(lens, dev([6, 9, 2]), table, free, n_free, q_start, slots, lens, n_free)
    assert lens.tolist() == [12, 11, 4] and status.item() == 11      # 1 block, 2, 1 of two: the last two are refused
    status.zero_()
    c.keep(table, lens, q_start, dev([[1, 4], [0, 8], [1, -1]]), dev([2, 2, 1]), change, slots=slots)
    tab = table.tolist()
    for a, b in ((6 + 1, 6), (6 + 4, 7)):
        ref.values[:, :, tab[0][b // block], b % block] = ref.values[:, :, tab[0][a // block], a % block]
    assert change.tolist() == [2 - 6, 0, 0] and status.item() == 0
    same(arena, None, ref)


@pytest.mark.parametrize("slots,nodes_there", [
    ([9] * 5 + [-1] * 8, False), ([9] * 5 + [-1] * 7 + [3], True), ([9] * 5 + [5] + [-1] * 7, True), ([9] * 13, True), ([-1] * 5 + [0] * 8, True),
    ([9] * 5, False), ([9] * 6, True), ([9] * 5 + [-1] * 8 + [9] * 4, False), ([], False)])
def test_which_slots_count(slots, nodes_there):
    """Any slot among the second sequence's eight nodes; those of other sequences, and what is beyond the array, do not."""
    ref = filled(np.random.default_rng(4), (1, 5, 8, 2), 64, "f16", True)
    c, arena, _ = device_cache(ref)
    tab, change = [[0, -1, -1], [3, 1, 4]], dev([7, 7])
    c.keep(dev(tab), dev([6, 20]), dev([0, 5, 13]), dev([[0, 1, 2], [1, 3, 5]]), dev([3, 3]), change, slots=dev(slots, np.int64))
    old = ref.values.copy()
    for place, node in enumerate((1, 3, 5) if nodes_there else ()):
        a, b = 12 + node, 12 + place
        ref.values[:, :, tab[1][b // 8], b % 8] = old[:, :, tab[1][a // 8], a % 8]
    assert change.tolist() == [3 - 5 if max(slots[:5], default=-1) >= 0 else 0, 3 - 8 if nodes_there else 0]
    same(arena, None, ref)


def test_captured_drafting_goes_on_when_blocks_run_out():
    """Extend, append, keep, extend as one graph: in replays that refuse some sequences nobody looks in between, and what every
    sequence holds at the end is what it took in."""
    rng = np.random.default_rng(11)
    block, hkv, hd, pool, n, nodes = 4, 1, 64, 20, 4, 7
    ref = R.Cache(1, pool, block, hkv, hd, "bf16")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, arena, _ = device_cache(ref, status=status)
    lens, q_start, slots, change, n_free = dev([0] * n), dev([0] * (n + 1)), dev([0] * (n * nodes), np.int64), dev([0] * n), dev([pool])
    table, free, add = dev(np.full((n, 12), -1)), dev(np.arange(pool)), dev([nodes] * n)
    accepted, count = dev(np.full((n, 3), -1)), dev([0] * n)
    x = torch.zeros((2, n * nodes, hkv, hd), dtype=torch.bfloat16, device="cuda")
    starts2, slots2 = torch.zeros_like(q_start), torch.zeros_like(slots)

    def step():
        c.extend(lens, add, table, free, n_free, q_start, slots, lens, n_free, stream=torch.cuda.current_stream())
        c.append(0, x[0], x[1], slots, stream=torch.cuda.current_stream())
        c.keep(table, lens, q_start, accepted, count, change, stream=torch.cuda.current_stream(), slots=slots)
        c.extend(lens, change, table, free, n_free, starts2, slots2, lens, n_free, stream=torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    held, refused = [[] for _ in range(n)], 0
    for turn in range(12):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape)).to(torch.bfloat16))
        paths = [np.sort(rng.permutation(nodes)[:rng.integers(0, 4)]) for _ in range(n)]
        rows = np.full((n, 3), -1)
        for s, p in enumerate(paths):
            rows[s, :len(p)] = p
        accepted.copy_(dev(rows))
        count.copy_(dev([len(p) for p in paths]))
        status.zero_()
        was = lens.tolist()
        graph.replay()
        got = slots.view(n, nodes).tolist()
        for s, p in enumerate(paths):
            if max(got[s]) < 0:
                refused += 1
                assert lens[s].item() == was[s] and status.item() == 11
            else:
                held[s] += [x[:, s * nodes + i].clone() for i in p]
        assert lens.tolist() == [len(h) for h in held]
        assert n_free.item() == pool - sum(-(-len(h) // block) for h in held)
    assert refused > 3 and min(len(h) for h in held) > 0
    view, tab = arena.view(torch.bfloat16).view(2, pool, block, hkv, hd), table.tolist()
    for s in range(n):
        for j, want in enumerate(held[s]):
            assert torch.equal(view[:, tab[s][j // block], j % block], want)
