"""emoe_kv_attend_tree and emoe_kv_attend_window on the GPU against the 64-bit definition.

Tolerance of out: with u the half step of the 16-bit type (bf16 2^-8, f16 2^-11), the weights are
rounded once (at most u of sum p|v|), the result once (u of |o| <= sum p|v|), and a score error e
moves every weight by a factor e^(+-e), which is 2e of sum p|v| after the division: (2u + 2e) sum p|v|
in all, second orders covered by a factor 1.05.  The weights that meet an e4m3 cache have a smallest step besides (rows_ref).  lse: e and a few roundings of 32 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import rows_ref as RR
from test_gpu_serving_kv import TORCH, device_cache, filled

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LARGEST = {"bf16": 3.3e38, "f16": 65504.0}
TINY = {"bf16": 1e-30, "f16": 2.0 ** -25}   # half a step of the smallest numbers


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, dtype))).cuda()


def make_tables(rng, pool, block, lens, extra_columns=1):
    ids = list(rng.permutation(pool).astype(np.int32))
    table = np.full((len(lens), max([-(-n // block) for n in lens] + [0]) + extra_columns), -1, np.int32)
    for i, n in enumerate(lens):
        table[i, :-(-n // block)] = [ids.pop() for _ in range(-(-n // block))]
    return table


def tree_bits(rng, n, density=None):
    """Ancestors and itself in a random tree; or, with a density, any graph (rows without any bit among them)."""
    bits = np.zeros((n, n), bool)
    if density is not None:
        bits[:] = rng.random((n, n)) < density
        bits[rng.random(n) < 0.2] = False
        return bits
    for i in range(n):
        if i:
            bits[i] = bits[rng.integers(0, i)]
        bits[i, i] = True
    return bits


def setup(seed, kv, io, hm, block, hkv, group, hd, lens, counts):
    rng = np.random.default_rng(seed)
    pool = sum(-(-n // block) for n in lens) + 2
    ref = filled(rng, (2, pool, block, hkv), hd, kv, hm)
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(int)
    q = torch.from_numpy(rng.standard_normal((max(1, starts[-1]), hkv * group, hd)) * 2).to(TORCH[io]).cuda()
    return rng, ref, make_tables(rng, pool, block, lens), starts, q


def call(c, q, table, lens, starts, *, bits=None, window=None, sinks=0, max_q=None, layer=1, out=None, scale=None, extra_words=0, stream=None):
    """out and lse of a call whose outputs and workspace hold garbage before."""
    counts = np.diff(starts)
    max_q = max(1, int(counts.max(initial=0))) if max_q is None else max_q
    out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    args = dict(scale=scale, lse=lse, stream=stream)
    if bits is not None:
        words = -(-max_q // 32) + extra_words
        mask = np.full((q.shape[0], words), -1, np.int32)
        for s, b in enumerate(bits):
            full = np.ones((len(b), words * 32), bool)   # bits of nodes that do not exist are set
            full[:, :b.shape[1]] = b
            mask[starts[s]:starts[s + 1]] = RR.packed_bits(full, words)
        need = c.attend_tree_workspace_bytes(len(lens), q.shape[0], max_q, q.shape[1], table.shape[1])
        work = torch.full((max(1, need),), 0xff, dtype=torch.uint8, device="cuda")
        c.attend_tree(layer, q, out, dev(table), dev(lens), dev(starts), dev(mask), max_q, workspace=work, **args)
    else:
        need = c.attend_window_workspace_bytes(len(lens), q.shape[0], max_q, q.shape[1], table.shape[1], window, sinks)
        work = torch.full((max(1, need),), 0xff, dtype=torch.uint8, device="cuda")
        c.attend_window(layer, q, out, dev(table), dev(lens), dev(starts), max_q, window, sinks, workspace=work, **args)
    torch.cuda.synchronize()
    return out, lse


def compare(got, got_l, want, io):
    """Within the tolerance where the definition is finite, and not finite where it is not."""
    o, want_l, a, e, far = (x.cpu().numpy() for x in want)
    got, got_l = got.double().cpu().numpy(), got_l.double().cpu().numpy()
    fine = np.isfinite(o) & (np.abs(o) < LARGEST[io])
    tol = 1.05 * ((2 * HALF_STEP[io] + 2 * e[..., None]) * a + far) + TINY[io]
    off = np.where(fine, np.abs(got - np.where(fine, o, 0)) / np.where(fine, tol, 1), 0)
    assert (off <= 1).all(), "out: %.3g times the tolerance at %s" % (np.nanmax(off), np.unravel_index(np.nanargmax(off), off.shape))
    assert np.isfinite(got[~fine]).sum() == 0
    assert np.array_equal(np.isneginf(got_l), np.isneginf(want_l))
    fine = np.isfinite(want_l)
    assert (np.abs(got_l[fine] - want_l[fine]) <= e[fine] + 2.0 ** -21 * np.abs(want_l[fine]) + 2.0 ** -20).all()
    assert np.isfinite(got_l[~fine]).sum() == 0


def check(ref, c, q, table, lens, starts, sees, io, scale=None, layer=1, **kw):
    n = starts[-1]
    out, lse = call(c, q, table, lens, starts, scale=scale, layer=layer, **kw)
    want = RR.attend(ref, layer, q[:n].double(), table, lens, starts, sees, q.shape[2] ** -0.5 if scale is None else scale)
    compare(out[:n], lse[:n], want, io)
    return out, lse


WINDOWS = [
    # kv, io, hm, block, KV heads, group, hd, lengths, query tokens, window, sinks
    ("bf16", "bf16", False, 16, 1, 8, 128, [1], [1], 1, 0),                                   # one token that sees itself
    ("bf16", "bf16", False, 16, 2, 4, 128, [33, 5, 17, 2500], [1, 1, 1, 1], 100, 4),          # shorter and longer than the window
    ("bf16", "bf16", True, 16, 4, 8, 128, [700, 260, 31], [1, 1, 1], 257, 0),                 # no first tokens
    ("f16", "f16", False, 5, 2, 5, 64, [77, 1, 40], [3, 1, 40], 7, 3),                        # a group of 5, blocks of 5, a whole prompt
    ("f16", "f16", True, 1, 1, 3, 32, [9, 40, 100], [2, 0, 100], 20, 1),                      # blocks of one token, a sequence without query tokens
    ("bf16", "bf16", False, 24, 2, 8, 128, [300, 90, 400], [300, 5, 37], 64, 100),            # first tokens that reach into the windows
    ("bf16", "bf16", False, 16, 2, 1, 256, [170, 200], [70, 130], 33, 2),
    ("e4m3", "bf16", False, 16, 3, 1, 128, [130, 64, 129], [1, 64, 129], 50, 4),
    ("e4m3", "f16", True, 16, 1, 16, 128, [3000], [1], 1500, 4),
    ("e4m3", "bf16", True, 7, 2, 2, 64, [200, 150], [31, 150], 1, 5),                         # a window of one token
    ("e4m3", "f16", False, 16, 4, 4, 32, [50, 100], [50, 7], 1 << 30, 0),                     # no limit: causal
    ("e4m3", "bf16", False, 32, 1, 8, 256, [640, 64], [64, 64], 128, 16),
    ("bf16", "bf16", False, 16, 1, 4, 128, [900, 1300, 700, 2, 0], [500, 1, 129, 1, 0], 300, 4),  # pieces of prompts among single tokens, an empty sequence
    ("f16", "f16", True, 16, 2, 8, 64, [1100, 1500], [1100, 200], 512, 1),
    ("e4m3", "bf16", False, 16, 2, 4, 128, [1000, 800, 40], [600, 1, 40], 256, 4),
    ("bf16", "bf16", False, 64, 2, 1, 128, [1025, 600], [1025, 600], 200, 4),                 # a head each: a tile has many tokens
    ("bf16", "bf16", False, 16, 1, 8, 64, [5000], [300], 4096, 4),
]


@pytest.mark.parametrize("kv,io,hm,block,hkv,group,hd,lens,counts,window,sinks", WINDOWS)
def test_window(kv, io, hm, block, hkv, group, hd, lens, counts, window, sinks):
    rng, ref, table, starts, q = setup(hd + len(lens) + window % 97, kv, io, hm, block, hkv, group, hd, lens, counts)
    c, _, _ = device_cache(ref)
    sees = [RR.window_sees(n, m, window, sinks) for n, m in zip(lens, counts)]
    check(ref, c, q, table, lens, starts, sees, io, window=window, sinks=sinks)


TREES = [
    # kv, io, hm, block, KV heads, group, hd, lengths, nodes, density (None: trees)
    ("bf16", "bf16", False, 16, 1, 8, 128, [1], [1], None),
    ("bf16", "bf16", False, 16, 1, 8, 128, [2375], [8], None),
    ("bf16", "bf16", True, 16, 4, 8, 128, [700, 26, 331], [26, 26, 1], None),                 # nodes without a context
    ("f16", "f16", False, 5, 2, 5, 64, [77, 1, 40], [33, 1, 40], None),                       # more nodes than a word has bits
    ("f16", "f16", True, 1, 1, 3, 32, [9, 40, 100], [2, 0, 100], 0.3),                        # any graph, rows that see no node
    ("bf16", "bf16", False, 24, 2, 8, 128, [64, 90, 70], [64, 5, 70], 0.1),                   # rows that see nothing at all
    ("bf16", "bf16", False, 16, 2, 1, 256, [170, 200], [70, 13], None),
    ("e4m3", "bf16", False, 16, 3, 1, 128, [130, 64, 1290], [13, 64, 5], None),
    ("e4m3", "f16", True, 16, 1, 16, 128, [3000, 10], [9, 10], None),
    ("e4m3", "bf16", True, 7, 2, 2, 64, [200, 150], [31, 150], 0.5),
    ("e4m3", "f16", False, 16, 4, 4, 32, [50, 100], [50, 7], None),
    ("e4m3", "bf16", False, 32, 1, 8, 256, [640, 64], [64, 64], None),
    ("bf16", "bf16", False, 16, 2, 8, 128, [4000, 3000, 2001], [64, 64, 64], None),
    ("f16", "f16", True, 16, 2, 8, 64, [2100, 1500, 0], [20, 97, 0], None),
    ("e4m3", "bf16", False, 16, 2, 8, 128, [2000, 1800], [60, 3], None),
    ("bf16", "bf16", False, 16, 2, 1, 128, [1500, 2600], [300, 129], 0.7),
]


@pytest.mark.parametrize("kv,io,hm,block,hkv,group,hd,lens,counts,density", TREES)
def test_tree(kv, io, hm, block, hkv, group, hd, lens, counts, density):
    rng, ref, table, starts, q = setup(hd + len(lens) + lens[0], kv, io, hm, block, hkv, group, hd, lens, counts)
    c, _, _ = device_cache(ref)
    bits = [tree_bits(rng, n, density) for n in counts]
    sees = [RR.tree_sees(n, m, b) for n, m, b in zip(lens, counts, bits)]
    check(ref, c, q, table, lens, starts, sees, io, bits=bits, extra_words=len(lens) % 2)


def poison(rng, ref, table, lens, counts, block, per_sequence):
    """Infinities, values and (e4m3) scales that are not numbers at random tokens of the sequences, most of them near the query tokens, and
    everywhere outside them."""
    used = np.zeros(ref.dims[2] * block, bool)
    for s, n in enumerate(lens):
        for j in range(n):
            used[table[s, j // block] * block + j % block] = True
    flat = ref.values.reshape(ref.dims[0], 2, -1, ref.dims[4], ref.head_dim)
    flat[:, :, ~used] = np.nan
    if ref.kv_type == "e4m3":
        ref.bytes.reshape(ref.dims[0], 2, -1, ref.dims[4])[:, :, ~used] = 255
    for s, n in enumerate(lens):
        for i in range(per_sequence):
            j = n - 1 - int(rng.integers(0, min(n, 2 * counts[s] + 8)))
            b, o, h = table[s, j // block], j % block, int(rng.integers(0, ref.dims[4]))
            kind = i % 4
            if kind == 0:
                ref.values[:, 1, b, o, h, int(rng.integers(0, ref.head_dim))] = np.nan
            elif kind == 1 and ref.kv_type != "e4m3":
                ref.values[:, 1, b, o, h, int(rng.integers(0, ref.head_dim))] = -np.inf
            elif kind == 1:
                ref.bytes[:, 1, b, o, h] = 255
            elif kind == 2:
                ref.values[:, 0, b, o, h] = np.nan
            elif ref.kv_type == "e4m3":
                ref.bytes[:, 0, b, o, h] = 255
                ref.bytes[:, 1, b, (o + 1) % block, h] = 127 + 90   # a value far beyond the others, for who sees it


ODD = [("bf16", "bf16", False, 16, 2, 4, 128), ("f16", "f16", True, 16, 2, 8, 64), ("e4m3", "bf16", False, 16, 2, 4, 128), ("e4m3", "f16", True, 8, 2, 2, 64),
       ("bf16", "bf16", True, 8, 1, 2, 32), ("e4m3", "bf16", False, 16, 2, 1, 256)]


@pytest.mark.parametrize("counts", [[1, 1, 1], [13, 1, 40], [150, 129, 2]])
@pytest.mark.parametrize("kv,io,hm,block,hkv,group,hd", ODD)
def test_what_a_row_does_not_see_has_no_influence(kv, io, hm, block, hkv, group, hd, counts):
    lens = [600, 350, 41]
    rng, ref, table, starts, q = setup(hd + counts[0], kv, io, hm, block, hkv, group, hd, lens, counts)
    poison(rng, ref, table, lens, counts, block, 9)
    c, _, _ = device_cache(ref)
    sees = [RR.window_sees(n, m, 20, 2) for n, m in zip(lens, counts)]
    check(ref, c, q, table, lens, starts, sees, io, window=20, sinks=2)
    bits = [tree_bits(rng, n) for n in counts]
    sees = [RR.tree_sees(n, m, b) for n, m, b in zip(lens, counts, bits)]
    check(ref, c, q, table, lens, starts, sees, io, bits=bits)


def test_blocks_behind_the_window_are_not_read():
    lens, counts = [900, 431], [40, 1]
    rng, ref, table, starts, q = setup(5, "bf16", "bf16", False, 16, 2, 4, 128, lens, counts)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, _, _ = device_cache(ref, status=status)
    for s in range(2):
        table[s, 1:(lens[s] - counts[s] + 1 - 100) // 16] = 1 << 30
    sees = [RR.window_sees(n, m, 100, 16) for n, m in zip(lens, counts)]
    check(ref, c, q, table, lens, starts, sees, "bf16", window=100, sinks=16)
    assert status.item() == 0


@pytest.mark.parametrize("counts", [[1, 1], [30, 140]])
def test_blocks_outside_the_pool_are_left_out_and_reported(counts):
    lens = [300, 400]
    for bad in (-1, 1 << 30):
        rng, ref, table, starts, q = setup(6, "f16", "f16", False, 16, 2, 4, 128, lens, counts)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        c, _, _ = device_cache(ref, status=status)
        table[0, 17] = table[1, 3] = table[1, 24] = bad
        sees = [RR.window_sees(n, m, 1000, 0) for n, m in zip(lens, counts)]
        check(ref, c, q, table, lens, starts, sees, "f16", window=1000)
        assert status.item() == 4


@pytest.mark.parametrize("hd,group", [(128, 4), (64, 16), (32, 2)])
def test_rows_of_no_sequence_stay_as_they_were(hd, group):
    """Room behind the last sequence, sequences with more query tokens than max_q, starts outside the tokens."""
    lens, counts = [500, 700, 90], [60, 1, 33]
    rng, ref, table, starts, q = setup(hd, "bf16", "bf16", False, 16, 2, group, hd, lens, counts)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, _, _ = device_cache(ref, status=status)
    q = torch.cat([q, torch.full_like(q[:7], float("nan"))])
    sees = [RR.window_sees(n, m, 40, 2) for n, m in zip(lens, counts)]
    bits = [tree_bits(rng, n) for n in counts]
    for kw in (dict(window=40, sinks=2), dict(bits=bits)):
        out, lse = call(c, q, table, lens, starts, **kw)
        assert (out[starts[-1]:] == 5).all() and (lse[starts[-1]:] == 5).all()
    assert status.item() == 0
    full, _ = call(c, q, table, lens, starts, window=40, sinks=2)
    out, lse = call(c, q, table, lens, starts, window=40, sinks=2, max_q=34)
    rest = slice(34, 60)
    assert status.item() == 11 and (out[rest] == 5).all() and (lse[rest] == 5).all()
    want = RR.attend(ref, 1, q[:94].double(), table, lens, starts, sees, hd ** -0.5)
    keep = [i for i in range(94) if not 34 <= i < 60]
    compare(out[keep], lse[keep], [x[keep] for x in want], "bf16")
    beyond = np.array([-5, 60, 61, 1 << 30])
    out, lse = call(c, q, table, lens, beyond, window=40, sinks=2, max_q=60)
    assert torch.equal(out[:61], full[:61])


def test_more_query_tokens_than_tokens():
    """Places before the first token see nothing; nodes of a tree see those that there are."""
    lens, counts = [3, 0], [6, 4]
    rng, ref, table, starts, q = setup(8, "bf16", "bf16", False, 16, 1, 4, 64, lens, counts)
    c, _, _ = device_cache(ref)
    check(ref, c, q, table, lens, starts, [RR.window_sees(n, m, 2, 1) for n, m in zip(lens, counts)], "bf16", window=2, sinks=1)
    bits = [tree_bits(rng, n, 0.6) for n in counts]
    check(ref, c, q, table, lens, starts, [RR.tree_sees(n, m, b) for n, m, b in zip(lens, counts, bits)], "bf16", bits=bits)


def test_strides_and_scales():
    lens, counts = [200, 333], [20, 150]
    rng, ref, table, starts, q = setup(9, "f16", "f16", False, 16, 2, 4, 128, lens, counts)
    c, _, _ = device_cache(ref)
    wide = torch.full((170, 3, 8, 128), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 1] = q
    outs = torch.full((170, 2, 8, 128), 7.0, dtype=torch.float16, device="cuda")
    sees = [RR.window_sees(n, m, 90, 0) for n, m in zip(lens, counts)]
    for scale in (0.02, -0.1, 0.0):
        check(ref, c, wide[:, 1], table, lens, starts, sees, "f16", scale=scale, window=90, out=outs[:, 0])
        assert (outs[:, 1] == 7).all()


def test_captured_with_lengths_that_change():
    """A captured call follows lengths, starts, tables and masks from replay to replay."""
    rng, ref, _, _, q = setup(10, "bf16", "bf16", False, 16, 2, 4, 128, [900, 900, 900], [30, 30, 30])
    c, _, _ = device_cache(ref)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    out2, lse2 = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    d_table, d_lens, d_starts = dev(np.zeros((3, 60))), dev([0, 0, 0]), dev([0, 0, 0, 0])
    d_mask = dev(np.zeros((90, 2)))
    work = [torch.empty(max(1, n), dtype=torch.uint8, device="cuda") for n in
            (c.attend_window_workspace_bytes(3, 90, 40, 8, 60, 200, 4), c.attend_tree_workspace_bytes(3, 90, 40, 8, 60))]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st = torch.cuda.current_stream()
        c.attend_window(1, q, out, d_table, d_lens, d_starts, 40, 200, 4, lse=lse, workspace=work[0], stream=st)
        c.attend_tree(1, q, out2, d_table, d_lens, d_starts, d_mask, 40, lse=lse2, workspace=work[1], stream=st)
    for lens, counts in (([900, 5, 333], [30, 5, 1]), ([40, 800, 0], [40, 2, 0]), ([1, 1, 1], [1, 1, 1]), ([930, 900, 900], [10, 40, 40])):
        table = make_tables(rng, ref.dims[2], 16, lens, 60 - max(-(-n // 16) for n in lens))
        starts = np.concatenate([[0], np.cumsum(counts)]).astype(int)
        bits = [tree_bits(rng, n) for n in counts]
        mask = np.zeros((90, 2), np.int32)
        for s, b in enumerate(bits):
            mask[starts[s]:starts[s + 1]] = RR.packed_bits(b, 2)
        for d, x in ((d_table, table), (d_lens, lens), (d_starts, starts), (d_mask, mask)):
            d.copy_(dev(x))
        graph.replay()
        torch.cuda.synchronize()
        n = starts[-1]
        for o, l, sees in ((out, lse, [RR.window_sees(*x, 200, 4) for x in zip(lens, counts)]), (out2, lse2, [RR.tree_sees(*x) for x in zip(lens, counts, bits)])):
            want = RR.attend(ref, 1, q[:n].double(), table, lens, starts, sees, 128 ** -0.5)
            compare(o[:n], l[:n], want, "bf16")


def test_the_same_results_on_another_stream_and_twice():
    lens, counts = [2000, 1500], [64, 3]
    rng, ref, table, starts, q = setup(11, "e4m3", "bf16", False, 16, 2, 8, 128, lens, counts)
    c, _, _ = device_cache(ref)
    bits = [tree_bits(rng, n) for n in counts]
    first, l1 = call(c, q, table, lens, starts, bits=bits)
    with torch.cuda.stream(torch.cuda.Stream()):
        second, l2 = call(c, q, table, lens, starts, bits=bits, stream=torch.cuda.current_stream())
    assert torch.equal(first, second) and torch.equal(l1, l2)


def test_a_shared_prefix_joined_by_lse():
    """A prefix through attend, own tokens through attend_tree, joined as documented."""
    lens, counts, block = [120, 90], [7, 7], 16
    rng, ref, table, starts, q = setup(12, "bf16", "bf16", False, block, 2, 4, 128, lens, counts)
    c, _, _ = device_cache(ref)
    prefix = np.array([table[0, 0], table[1, 1], table[0, 3]], np.int32)
    o1, l1 = torch.empty_like(q).view(2, 7, 8, 128), torch.empty((2, 7, 8), device="cuda")
    work = torch.empty(max(1, c.attend_workspace_bytes(2, 7, 8, 0, 41)), dtype=torch.uint8, device="cuda")
    c.attend(1, q.view(2, 7, 8, 128), o1, None, None, dev(prefix), 41, lse=l1, workspace=work)
    bits = [tree_bits(rng, n) for n in counts]
    o2, l2 = call(c, q, table, lens, starts, bits=bits)
    both = torch.stack([l1.view(14, 8), l2]).double()
    w = torch.softmax(both, 0)[..., None]
    got = w[0] * o1.view(14, 8, 128).double() + w[1] * o2.double()
    long = [np.concatenate([prefix, t]) for t in table]
    # the prefix ends inside a block: its tokens and the own ones as one sequence, by hand
    want, a = torch.zeros_like(got), torch.zeros_like(got)
    flat = torch.from_numpy(ref.values[1].reshape(2, -1, 2, 128)).cuda()
    for s in range(2):
        at = [prefix[j // block] * block + j % block for j in range(41)] + [table[s][j // block] * block + j % block for j in range(lens[s])]
        k, v = flat[0, at], flat[1, at]
        see = torch.from_numpy(np.concatenate([np.ones((7, 41), bool), RR.tree_sees(lens[s], 7, bits[s])], 1)).cuda()
        for h in range(8):
            p = torch.softmax((q[7 * s:7 * s + 7, h].double() @ k[:, h // 4].T * 128 ** -0.5).masked_fill(~see, float("-inf")), -1)
            want[7 * s:7 * s + 7, h], a[7 * s:7 * s + 7, h] = p @ v[:, h // 4], p @ v[:, h // 4].abs()
    assert long and ((got - want).abs() <= (2.2 * 2.0 ** -8 + 1e-3) * a).all()


def test_offsets_beyond_32_bits():
    """A cache of 8.6 GB a layer whose used blocks lie at its end."""
    block, heads, hd, pool = 64, 8, 128, 65600
    arena = torch.zeros(2 * pool * block * heads * hd, dtype=torch.bfloat16, device="cuda")
    c = E.KvCache(arena.view(torch.uint8), n_layers=1, num_blocks=pool, block_tokens=block, n_heads=heads, head_dim=hd)
    rng = np.random.default_rng(3)
    last = rng.standard_normal((2, 16, block, heads, hd))
    view = arena.view(2, pool, block, heads, hd)
    view[:, -16:] = torch.from_numpy(last).to(torch.bfloat16).cuda()
    ref = filled(rng, (1, 16, block, heads), hd, "bf16", False)
    ref.values[0] = view[:, -16:].double().cpu().numpy()
    small = np.array([[3, 9, 0, 15, 7], [8, 2, 11, 1, -1]], np.int32)
    table = np.where(small < 0, -1, small + pool - 16).astype(np.int32)
    lens, counts = [300, 250], [40, 1]
    starts = np.array([0, 40, 41])
    q = torch.from_numpy(rng.standard_normal((41, 16, hd)) * 2).to(torch.bfloat16).cuda()
    sees = [RR.window_sees(n, m, 150, 4) for n, m in zip(lens, counts)]
    out, lse = call(c, q, table, lens, starts, window=150, sinks=4, layer=0)
    compare(out, lse, RR.attend(ref, 0, q.double(), small, lens, starts, sees, hd ** -0.5), "bf16")


MANY = [("bf16", "bf16", False, 16, 2, 8, 128), ("f16", "f16", True, 16, 4, 8, 64), ("e4m3", "bf16", False, 16, 2, 8, 128), ("e4m3", "f16", True, 8, 4, 8, 64),
        ("bf16", "bf16", True, 24, 12, 1, 128), ("f16", "f16", False, 16, 5, 3, 128)]


@pytest.mark.parametrize("kv,io,hm,block,hkv,group,hd", MANY)
def test_what_many_rows_do_not_see_has_no_influence(kv, io, hm, block, hkv, group, hd):
    """As above at sizes that go to the tensor core kernel: pieces of prompts, and trees, of many rows beside small ones."""
    lens, counts = [1500, 900, 700, 130], [400, 129, 2, 130]
    rng, ref, table, starts, q = setup(hd + group, kv, io, hm, block, hkv, group, hd, lens, counts)
    poison(rng, ref, table, lens, counts, block, 30)
    c, _, _ = device_cache(ref)
    sees = [RR.window_sees(n, m, 450, 130) for n, m in zip(lens, counts)]
    check(ref, c, q, table, lens, starts, sees, io, window=450, sinks=130)
    bits = [tree_bits(rng, n, 0.5 if n == 129 else None) for n in counts]
    sees = [RR.tree_sees(n, m, b) for n, m, b in zip(lens, counts, bits)]
    check(ref, c, q, table, lens, starts, sees, io, bits=bits)


MORE = [
    # kv, io, hm, block, KV heads, group, hd, lengths, query tokens, window, sinks: many rows
    ("bf16", "bf16", False, 16, 1, 1, 128, [2300], [2300], 600, 4),                          # a whole prompt, tiles of 256 tokens
    ("bf16", "bf16", False, 16, 2, 2, 64, [3000, 2600], [1000, 900], 1 << 30, 0),             # causal
    ("f16", "f16", True, 32, 2, 8, 128, [2500, 640, 1900], [17, 600, 1], 1000, 300),          # 136 rows, many, 8 of them
    ("e4m3", "bf16", False, 16, 2, 4, 128, [2300, 700], [300, 700], 130, 4),                  # windows about as long as a tile
    ("e4m3", "f16", True, 16, 2, 5, 64, [5000], [200], 2000, 1),
    ("bf16", "bf16", False, 16, 8, 8, 128, [1100] * 20, [3] * 20, 900, 4),                    # 24 rows each
    ("bf16", "bf16", False, 16, 4, 8, 128, [1300] + [700] * 40, [300] + [1] * 40, 500, 4),    # single tokens beside a piece
    ("f16", "f16", False, 16, 1, 16, 128, [20000], [16], 1 << 30, 0),                         # split over the tokens
    ("bf16", "bf16", False, 16, 1, 8, 128, [9000, 300], [16, 300], 8000, 77),
]


@pytest.mark.parametrize("kv,io,hm,block,hkv,group,hd,lens,counts,window,sinks", MORE)
def test_window_with_many_rows(kv, io, hm, block, hkv, group, hd, lens, counts, window, sinks):
    rng, ref, table, starts, q = setup(hd + len(lens) + window % 97, kv, io, hm, block, hkv, group, hd, lens, counts)
    c, _, _ = device_cache(ref)
    sees = [RR.window_sees(n, m, window, sinks) for n, m in zip(lens, counts)]
    check(ref, c, q, table, lens, starts, sees, io, window=window, sinks=sinks)


@pytest.mark.parametrize("hd,kv", [(128, "bf16"), (64, "e4m3")])
def test_waits_that_run_out_are_reported(hd, kv):
    lens, counts = [3000], [200]
    rng, ref, table, starts, q = setup(1, kv, "bf16", False, 16, 2, 8, hd, lens, counts)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, _, _ = device_cache(ref, status=status)
    need = c.attend_window_workspace_bytes(1, 200, 200, 16, table.shape[1], 2000, 0)
    args = (1, q, torch.empty_like(q), dev(table), dev(lens), dev(starts), 200, 2000)
    work = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
    c.attend_window(*args, workspace=work, wait_limit_us=-1)
    torch.cuda.synchronize()
    assert status.item() == 10 and torch.isnan(args[2]).any()
    status.zero_()
    check(ref, c, q, table, lens, starts, [RR.window_sees(3000, 200, 2000, 0)], "bf16", window=2000)
    assert status.item() == 0


@pytest.mark.parametrize("kv,io,hd", [("bf16", "bf16", 128), ("f16", "f16", 64), ("e4m3", "bf16", 128), ("e4m3", "f16", 64)])
def test_scales_and_strides_with_many_rows(kv, io, hd):
    """Any finite scale, rows of wider tensors, at sizes for the tensor core kernel: a whole tile of rows and half a one."""
    lens, counts = [1900, 1400], [200, 9]
    rng, ref, table, starts, q = setup(hd, kv, io, False, 16, 2, 8, hd, lens, counts)
    c, _, _ = device_cache(ref)
    wide = torch.full((209, 2, 16, hd), float("nan"), dtype=TORCH[io], device="cuda")
    wide[:, 1] = q
    outs = torch.full((209, 2, 16, hd), 7.0, dtype=TORCH[io], device="cuda")
    sees = [RR.window_sees(n, m, 1000, 4) for n, m in zip(lens, counts)]
    bits = [tree_bits(rng, n) for n in counts]
    for scale in (0.05, -0.07, 0.0):
        check(ref, c, wide[:, 1], table, lens, starts, sees, io, scale=scale, window=1000, sinks=4, out=outs[:, 0])
        check(ref, c, wide[:, 1], table, lens, starts, [RR.tree_sees(*x) for x in zip(lens, counts, bits)], io, scale=scale, bits=bits, out=outs[:, 0])
        assert (outs[:, 1] == 7).all()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_more_query_tokens_than_tokens_with_many_rows(kv):
    lens, counts = [100, 1700, 3], [300, 260, 150]
    rng, ref, table, starts, q = setup(13, kv, "bf16", False, 16, 4, 8, 128, lens, counts)
    c, _, _ = device_cache(ref)
    check(ref, c, q, table, lens, starts, [RR.window_sees(n, m, 1500, 4) for n, m in zip(lens, counts)], "bf16", window=1500, sinks=4)
    bits = [tree_bits(rng, n, 0.4) for n in counts]
    check(ref, c, q, table, lens, starts, [RR.tree_sees(n, m, b) for n, m, b in zip(lens, counts, bits)], "bf16", bits=bits)


def test_on_three_streams_at_once():
    """Calls of every kernel, each with a workspace of its own, give what they give alone."""
    cases = []
    for seed, (lens, counts) in enumerate((([3000, 2500], [200, 40]), ([1500] * 40, [1] * 40), ([2000, 900, 700], [2, 2, 1]))):
        rng, ref, table, starts, q = setup(20 + seed, "bf16", "bf16", False, 16, 4, 8, 128, lens, counts)
        c, _, _ = device_cache(ref)
        want = call(c, q, table, lens, starts, window=1200, sinks=4)
        need = c.attend_window_workspace_bytes(len(lens), q.shape[0], max(counts), 32, table.shape[1], 1200, 4)
        cases.append((c, q, torch.empty_like(q), torch.empty(q.shape[:2], device="cuda"), dev(table), dev(lens), dev(starts), max(counts),
                      torch.empty(max(1, need), dtype=torch.uint8, device="cuda"), torch.cuda.Stream(), want))
    torch.cuda.synchronize()
    for _ in range(5):
        for c, q, out, lse, table, lens, starts, max_q, work, st, _ in cases:
            c.attend_window(1, q, out, table, lens, starts, max_q, 1200, 4, lse=lse, workspace=work, stream=st)
    torch.cuda.synchronize()
    for _, _, out, lse, _, _, _, _, _, _, want in cases:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_prompts_in_pieces_then_single_tokens():
    """Extend, append, attend_window step by step: pieces of prompts among sequences that decode, blocks behind the window given to nobody."""
    rng = np.random.default_rng(14)
    block, hkv, hd, pool, window, sinks = 8, 2, 128, 60, 50, 3
    c, arena, _ = device_cache(filled(rng, (1, pool, block, hkv), hd, "bf16", False))
    n, lens, q_start, n_free = 3, dev([0] * 3), dev([0] * 4), dev([pool])
    table, free, slots = dev(np.full((n, 24), -1)), dev(rng.permutation(pool)), dev(np.zeros(128), np.int64)
    kept = [[], [], []]
    for add in ([40, 5, 33], [30, 1, 40], [1, 1, 40], [1, 1, 20], [1, 1, 1], [0, 1, 1]):
        c.extend(lens, dev(add), table, free, n_free, q_start, slots, lens, n_free)
        x = torch.from_numpy(rng.standard_normal((2, 128, hkv, hd))).to(torch.bfloat16).cuda()
        c.append(0, x[0], x[1], slots)
        q = torch.from_numpy(rng.standard_normal((128, 8, hd))).to(torch.bfloat16).cuda()
        out = torch.empty_like(q)
        work = torch.empty(max(1, c.attend_window_workspace_bytes(n, 128, 40, 8, 24, window, sinks)), dtype=torch.uint8, device="cuda")
        c.attend_window(0, q, out, table, lens, q_start, 40, window, sinks, workspace=work)
        at = q_start.tolist()
        for s in range(n):
            kept[s] += [x[:, i] for i in range(at[s], at[s + 1])]
            seq = torch.stack(kept[s], 1).double()
            see = torch.from_numpy(RR.window_sees(len(kept[s]), add[s], window, sinks)).cuda()
            for h in range(8):
                p = torch.softmax((q[at[s]:at[s + 1], h].double() @ seq[0, :, h // 4].T * hd ** -0.5).masked_fill(~see, float("-inf")), -1)
                want, a = p @ seq[1, :, h // 4], p @ seq[1, :, h // 4].abs()
                assert ((out[at[s]:at[s + 1], h].double() - want).abs() <= 2.2 * 2.0 ** -8 * a).all()
    assert lens.tolist() == [len(k) for k in kept]


@pytest.mark.parametrize("kv,io,group", [("e4m3", "bf16", 1), ("bf16", "bf16", 4), ("f16", "f16", 1)])
def test_many_sequences_of_different_lengths(kv, io, group):
    """More blocks than run at once: the longest sequences come first, equal ones and empty ones among them."""
    lens = [int(x) for x in np.random.default_rng(1).integers(0, 300, 60)] + [300, 300, 0, 0, 17]
    counts = [min(n, 1 + i % (13 if group == 1 else 3)) for i, n in enumerate(lens)]
    rng, ref, table, starts, q = setup(15 + group, kv, io, group == 4, 16, 8, group, 64, lens, counts)
    c, _, _ = device_cache(ref)
    bits = [tree_bits(rng, n) for n in counts]
    check(ref, c, q, table, lens, starts, [RR.tree_sees(n, m, b) for n, m, b in zip(lens, counts, bits)], io, bits=bits)
    check(ref, c, q, table, lens, starts, [RR.window_sees(n, m, 1 << 30, 0) for n, m in zip(lens, counts)], io, window=1 << 30)


@pytest.mark.parametrize("kv,io", [("bf16", "bf16"), ("e4m3", "f16")])
def test_many_trees_of_different_lengths(kv, io):
    """As above on the tensor core kernel: more blocks than SMs."""
    lens = [int(x) for x in np.random.default_rng(2).integers(0, 700, 40)] + [700, 700, 0, 9]
    counts = [min(n, 10 + i % 11) for i, n in enumerate(lens)]
    rng, ref, table, starts, q = setup(17, kv, io, False, 16, 4, 8, 64, lens, counts)
    c, _, _ = device_cache(ref)
    bits = [tree_bits(rng, n) for n in counts]
    check(ref, c, q, table, lens, starts, [RR.tree_sees(n, m, b) for n, m, b in zip(lens, counts, bits)], io, bits=bits)
    check(ref, c, q, table, lens, starts, [RR.window_sees(n, m, 1 << 30, 0) for n, m in zip(lens, counts)], io, window=1 << 30)
