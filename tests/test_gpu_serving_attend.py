"""emoe_kv_attend on the GPU against the 64-bit definition.

Tolerance of out: with u the half step of the 16-bit type (bf16 2^-8, f16 2^-11), the weights are
rounded once (at most u of sum p|v|), the result once (u of |o| <= sum p|v|), and a score error e
moves every weight by a factor e^(+-e), which is 2e of sum p|v| after the division: (2u + 2e) sum p|v|
in all, e from serving_ref.attend, second orders covered by a factor 1.05.  lse: e and a few roundings of 32 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import serving_ref as R
from test_gpu_serving_kv import TORCH, device_cache, filled

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def make_tables(rng, pool, block, prefix, lens, extra_columns=0):
    ids = list(rng.permutation(pool).astype(np.int32))
    take = lambda n: [ids.pop() for _ in range(n)]    # noqa: E731
    pt = np.array(take(-(-prefix // block)), np.int32)
    width = max([-(-n // block) for n in lens] + [0]) + extra_columns
    table = np.full((len(lens), width), -1, np.int32)
    for i, n in enumerate(lens):
        table[i, :-(-n // block)] = take(-(-n // block))
    return pt, table


def check(ref, c, q, pt, prefix, table, lens, io, scale=None, layer=0, out=None, lse=True, stream=None):
    n, t, hq, hd = q.shape
    dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()    # noqa: E731
    out = torch.full(q.shape, 5.0, dtype=TORCH[io], device="cuda") if out is None else out
    l = torch.full((n, t, hq), 5.0, device="cuda") if lse else None
    width = 0 if table is None else table.shape[1]
    work = torch.full((max(1, c.attend_workspace_bytes(n, t, hq, width, prefix)),), 0xff, dtype=torch.uint8, device="cuda")
    c.attend(layer, q, out, dev(table), None if table is None else dev(np.asarray(lens, np.int32)), dev(pt) if prefix else None, prefix,
             scale=scale, lse=l, workspace=work, stream=stream)
    torch.cuda.synchronize()
    scale = hd ** -0.5 if scale is None else scale
    if table is None:
        table, lens = np.zeros((n, 0), np.int32), [0] * n
    o, want_l, a, e = R.attend(ref, layer, q.double().cpu().numpy(), table, lens, pt, prefix, scale)
    got = out.double().cpu().numpy()
    tol = 1.05 * (2 * HALF_STEP[io] + 2 * e[..., None]) * a + 1e-30
    off = np.abs(got - o) / tol
    assert (off <= 1).all(), "out: %.3g times the tolerance at %s" % (np.nanmax(off), np.unravel_index(np.nanargmax(off), off.shape))
    if lse:
        got_l = l.double().cpu().numpy()
        assert np.array_equal(np.isinf(got_l), np.isinf(want_l))
        fine = np.isfinite(want_l)
        assert (np.abs(got_l - want_l)[fine] <= e[fine] + 2.0 ** -21 * np.abs(want_l[fine]) + 2.0 ** -20).all()
    return out


CASES = [
    # kv, io, hm, block, hkv, group, hd, q_len, prefix, own lengths
    ("bf16", "bf16", False, 16, 1, 8, 128, 1, 0, [1]),                       # one token of one sequence
    ("bf16", "bf16", False, 16, 2, 4, 128, 1, 0, [33, 0, 17, 250]),          # an empty sequence among others
    ("bf16", "bf16", True, 16, 4, 8, 128, 1, 200, [16, 15, 31]),
    ("f16", "f16", False, 5, 2, 5, 64, 1, 37, [7, 1]),                       # a group of 5, blocks of 5
    ("f16", "f16", True, 1, 1, 3, 32, 2, 9, [2, 40, 1]),                     # blocks of one token; a row before the first own token
    ("bf16", "bf16", False, 24, 2, 8, 128, 5, 0, [3, 90, 5]),                # 40 rows a sequence; rows that see nothing
    ("bf16", "bf16", False, 16, 2, 1, 256, 1, 65, [70, 200]),
    ("e4m3", "bf16", False, 16, 3, 1, 128, 1, 130, [1, 64, 129]),
    ("e4m3", "f16", True, 16, 1, 16, 128, 1, 0, [300]),
    ("e4m3", "bf16", True, 7, 2, 2, 64, 3, 22, [2, 50]),
    ("e4m3", "f16", False, 16, 4, 4, 32, 1, 0, [5, 100]),
    ("e4m3", "bf16", False, 32, 1, 8, 256, 1, 64, [64]),
    ("bf16", "bf16", False, 16, 2, 2, 128, 1, 1500, [0, 0, 0]),              # the prefix alone
    ("bf16", "bf16", False, 16, 1, 4, 128, 1, 1, [1] * 37),                  # more rows than a tile, a prefix of one token
]


@pytest.mark.parametrize("kv,io,hm,block,hkv,group,hd,t,prefix,lens", CASES)
def test_attend(kv, io, hm, block, hkv, group, hd, t, prefix, lens):
    rng = np.random.default_rng(hd + prefix + len(lens))
    pool = -(-prefix // block) + sum(-(-n // block) for n in lens) + 2
    ref = filled(rng, (2, pool, block, hkv), hd, kv, hm)
    c, arena, scales = device_cache(ref)
    pt, table = make_tables(rng, pool, block, prefix, lens, extra_columns=1)
    q = torch.from_numpy(rng.standard_normal((len(lens), t, hkv * group, hd)) * 2).to(TORCH[io]).cuda()
    check(ref, c, q, pt, prefix, table, lens, io, layer=1)


def test_no_token_at_all():
    rng = np.random.default_rng(1)
    ref = filled(rng, (1, 2, 4, 2), 64, "bf16", False)
    c, _, _ = device_cache(ref)
    q = torch.randn(3, 1, 4, 64, device="cuda", dtype=torch.bfloat16)
    out = check(ref, c, q, np.zeros(0, np.int32), 0, None, None, "bf16")
    assert not out.any()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_what_lies_behind_the_length_has_no_influence(kv):
    """NaN and infinities in the rest of the last blocks, in unused blocks, and - for the earlier of two
    query tokens - in the last token itself."""
    rng = np.random.default_rng(2)
    lens, prefix, block = [20, 3, 17], 21, 16
    ref = filled(rng, (1, 12, block, 2), 64, kv, False)
    pt, table = make_tables(rng, 12, block, prefix, lens, extra_columns=2)
    clean = device_cache(ref)[0]
    used = np.zeros((12, block), bool)
    for j in range(prefix):
        used[pt[j // block], j % block] = True
    for s, n in enumerate(lens):
        for j in range(n - 1):
            used[table[s, j // block], j % block] = True
    c, arena, scales = device_cache(ref)
    bad = torch.from_numpy(~used).cuda()
    if kv == "bf16":
        arena.view(torch.bfloat16).view(1, 2, 12, block, 2, 64)[:, :, bad] = float("nan")
    else:
        arena.view(1, 2, 12, block, 2, 64)[:, :, bad] = 0x7f
        scales[:, :, bad] = 255
    q = torch.randn(3, 2, 4, 64, device="cuda", dtype=torch.bfloat16)
    dev = [torch.from_numpy(x).cuda() for x in (table, np.array(lens, np.int32), pt)]
    outs = []
    for cache in (clean, c):
        out = torch.empty_like(q)
        work = torch.empty(cache.attend_workspace_bytes(3, 2, 4, table.shape[1], prefix), dtype=torch.uint8, device="cuda")
        cache.attend(0, q, out, dev[0], dev[1], dev[2], prefix, workspace=work)
        outs.append(out)
    assert torch.equal(outs[0][:, 0], outs[1][:, 0])        # the first query token does not see the last one
    assert torch.isnan(outs[1][:, 1]).all()                 # the second does: loudly


def test_blocks_outside_the_pool_are_left_out_and_reported():
    rng = np.random.default_rng(3)
    lens, prefix, block = [40, 9], 33, 8
    ref = filled(rng, (1, 14, block, 2), 128, "bf16", False)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, _, _ = device_cache(ref, status=status)
    pt, table = make_tables(rng, 14, block, prefix, lens)
    q = torch.randn(2, 1, 4, 128, device="cuda", dtype=torch.bfloat16)
    check(ref, c, q, pt, prefix, table, lens, "bf16")
    assert status.item() == 0
    table[0, 1], table[0, 4], pt[2] = 14, -5, 1 << 30
    check(ref, c, q, pt, prefix, table, lens, "bf16")
    assert status.item() == 4


def test_lengths_beyond_the_table_count_as_its_size():
    rng = np.random.default_rng(4)
    ref = filled(rng, (1, 6, 8, 1), 64, "f16", False)
    c, _, _ = device_cache(ref)
    table = np.array([[0, 3], [2, 5]], np.int32)
    q = torch.randn(2, 1, 2, 64, device="cuda", dtype=torch.float16)
    check(ref, c, q, np.zeros(0, np.int32), 0, table, [1 << 30, -7], "f16")


def test_large_scores_and_equal_scores():
    """Scores of a few hundred (the maximum has to be taken out), and all equal ones."""
    rng = np.random.default_rng(6)
    ref = filled(rng, (1, 40, 16, 1), 64, "bf16", False)
    c, _, _ = device_cache(ref)
    pt, table = make_tables(rng, 40, 16, 100, [300, 150])
    q = torch.randn(2, 1, 4, 64, device="cuda", dtype=torch.bfloat16)
    for scale in (8.0, 0.0, -4.0, 2.0 ** -20):
        check(ref, c, q, pt, 100, table, [300, 150], "bf16", scale=scale)


def test_strided_queries_and_outputs():
    """q as a part of a fused projection's output, out into a wider tensor whose rest stays."""
    rng = np.random.default_rng(7)
    ref = filled(rng, (1, 9, 16, 2), 64, "f16", False)
    c, _, _ = device_cache(ref)
    pt, table = make_tables(rng, 9, 16, 10, [40, 20])
    wide = torch.randn(2, 3, 12, 64, device="cuda", dtype=torch.float16)
    target = torch.full((2, 3, 6, 64), 9.0, device="cuda", dtype=torch.float16)
    check(ref, c, wide[:, :, 2:6], pt, 10, table, [40, 20], "f16", out=target[:, :, 1:5])
    assert bool((target[:, :, 0] == 9).all()) and bool((target[:, :, 5] == 9).all())


def test_captured_call_follows_lengths_and_tables():
    rng = np.random.default_rng(8)
    ref = filled(rng, (1, 30, 16, 2), 128, "e4m3", False)
    c, _, _ = device_cache(ref)
    pt, table = make_tables(rng, 30, 16, 50, [60, 60, 60])
    q = torch.randn(3, 1, 8, 128, device="cuda", dtype=torch.bfloat16)
    out = torch.empty_like(q)
    d_table, d_pt = torch.from_numpy(table).cuda(), torch.from_numpy(pt).cuda()
    lens = torch.tensor([1, 1, 1], dtype=torch.int32, device="cuda")
    work = torch.empty(c.attend_workspace_bytes(3, 1, 8, table.shape[1], 50), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.attend(0, q, out, d_table, lens, d_pt, 50, workspace=work, stream=side)
    for now in ([1, 60, 0], [17, 2, 33]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        assert torch.equal(check(ref, c, q, pt, 50, table, now, "bf16"), first)     # and the same bits each time


def test_parts_are_joined_with_lse():
    """Two calls over halves of a context, joined as documented, agree with one call."""
    rng = np.random.default_rng(9)
    ref = filled(rng, (1, 16, 16, 1), 64, "f16", False)
    c, _, _ = device_cache(ref)
    table = np.arange(16, dtype=np.int32)[None]
    q = torch.randn(1, 1, 4, 64, device="cuda", dtype=torch.float16)
    whole, lse = torch.empty_like(q), torch.empty(1, 1, 4, device="cuda")

    def call(t, n):
        out, l = torch.empty_like(q), torch.empty(1, 1, 4, device="cuda")
        w = torch.empty(c.attend_workspace_bytes(1, 1, 4, t.shape[1]) + 1, dtype=torch.uint8, device="cuda")
        c.attend(0, q, out, torch.from_numpy(t).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), lse=l, workspace=w)
        return out.double(), l.double()[..., None]

    whole, lse = call(table, 250)
    (o1, l1), (o2, l2) = call(table[:, :8].copy(), 128), call(table[:, 8:].copy(), 122)
    joined = (o1 * l1.exp() + o2 * l2.exp()) / (l1.exp() + l2.exp())
    # |v| <= 5 here: three results rounded to f16, half a step each, of sums of magnitudes of at most 5
    assert (joined - whole).abs().max().item() <= 4 * 2.0 ** -11 * 5 + 1e-4
    assert (torch.log(l1.exp() + l2.exp()) - lse).abs().max().item() < 1e-4


def test_two_streams_with_workspaces_of_their_own():
    rng = np.random.default_rng(10)
    ref = filled(rng, (1, 64, 16, 2), 128, "bf16", False)
    c, _, _ = device_cache(ref)
    pt, table = make_tables(rng, 64, 16, 300, [200, 100])
    dev = [torch.from_numpy(x).cuda() for x in (table, np.array([200, 100], np.int32), pt)]
    q = torch.randn(2, 1, 8, 128, device="cuda", dtype=torch.bfloat16)
    want = check(ref, c, q, pt, 300, table, [200, 100], "bf16")
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty(20, *q.shape, dtype=q.dtype, device="cuda") for _ in range(2)]
    works = [torch.empty(c.attend_workspace_bytes(2, 1, 8, table.shape[1], 300), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for s in range(2):
            c.attend(0, q, outs[s][i], dev[0], dev[1], dev[2], 300, workspace=works[s], stream=streams[s])
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(x, want) for x in o)
