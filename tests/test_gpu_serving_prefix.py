"""emoe_kv_attend where a prefix meets several row tiles, against the 64-bit definition with the tolerance of
test_gpu_serving_attend.  Most are small enough for the row kernel; test_gpu_serving_prefix_wide has the same with
the work that goes to the 5th-generation tensor core path."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import serving_ref as R
from test_gpu_serving_attend import check, make_tables
from test_gpu_serving_kv import TORCH, device_cache, filled

pytestmark = pytest.mark.gpu

CASES = [
    # kv, io, hm, block, hkv, group, hd, q_len, prefix, sequences
    ("bf16", "bf16", False, 16, 1, 8, 128, 1, 128, 3),       # one tile: the second slot has none
    ("bf16", "bf16", False, 16, 1, 1, 128, 1, 129, 17),      # two tiles, one row above the small path
    ("bf16", "bf16", True, 16, 2, 4, 128, 1, 700, 32),       # 128 rows, odd number of tiles
    ("f16", "f16", False, 5, 2, 3, 64, 1, 333, 20),          # blocks of 5
    ("f16", "f16", True, 1, 1, 16, 64, 2, 260, 5),           # 160 rows: two row tiles
    ("bf16", "bf16", False, 24, 3, 8, 128, 1, 1000, 32),     # exactly 256 rows
    ("bf16", "bf16", False, 16, 1, 8, 64, 3, 513, 13),       # 312 rows: a second block with one row tile
    ("f16", "f16", False, 16, 1, 8, 128, 1, 2000, 70),       # 560 rows, several splits
    ("e4m3", "bf16", False, 16, 2, 1, 128, 1, 1111, 33),
    ("e4m3", "bf16", True, 7, 1, 8, 64, 1, 300, 20),
    ("e4m3", "f16", False, 16, 1, 8, 128, 2, 400, 17),
    ("e4m3", "f16", True, 16, 2, 2, 64, 1, 129, 40),
    ("bf16", "bf16", False, 16, 1, 32, 128, 1, 1, 2),        # a prefix of one token
    ("e4m3", "bf16", False, 16, 1, 4, 128, 1, 3, 80),
]


@pytest.mark.parametrize("kv,io,hm,block,hkv,group,hd,t,prefix,seqs", CASES)
@pytest.mark.parametrize("own", [True, False])
def test_prefix(kv, io, hm, block, hkv, group, hd, t, prefix, seqs, own):
    rng = np.random.default_rng(hd + prefix + seqs)
    lens = [int(x) for x in rng.integers(0, 20, seqs)] if own else [0] * seqs
    pool = -(-prefix // block) + sum(-(-n // block) for n in lens) + 2
    ref = filled(rng, (1, pool, block, hkv), hd, kv, hm)
    c, arena, scales = device_cache(ref)
    pt, table = make_tables(rng, pool, block, prefix, lens)
    q = torch.from_numpy(rng.standard_normal((seqs, t, hkv * group, hd)) * 2).to(TORCH[io]).cuda()
    if own:
        check(ref, c, q, pt, prefix, table, lens, io)
    else:
        check(ref, c, q, pt, prefix, None, None, io)


@pytest.mark.parametrize("kv,io", [("bf16", "bf16"), ("e4m3", "f16"), ("e4m3", "bf16")])
def test_scores_that_raise_the_maximum_and_signs(kv, io):
    """Keys that grow along the prefix (the maximum is raised again and again), shrinking ones, a negative,
    a zero and a tiny scale."""
    rng = np.random.default_rng(5)
    ref = R.Cache(1, 50, 16, 1, 64, kv)
    grow = np.linspace(0.05, 6, 800).reshape(50, 16)[None, None, :, :, None, None] ** 2
    x = rng.standard_normal(ref.values.shape) * grow
    if kv == "e4m3":
        ref.values, ref.bytes = R.quantise(x.astype(np.float32))
    else:
        ref.values = torch.from_numpy(x).to(TORCH[kv]).double().numpy()
    c, _, _ = device_cache(ref)
    for order in (np.arange(50), np.arange(50)[::-1]):
        pt = order.astype(np.int32)
        q = torch.from_numpy(rng.standard_normal((40, 1, 4, 64))).to(TORCH[io]).cuda()
        for scale in (0.125, -1.0, 0.0, 2.0 ** -30):
            check(ref, c, q, pt, 795, None, None, io, scale=scale)


@pytest.mark.parametrize("rows", [30, 4])
def test_small_and_large_values_in_e4m3_with_f16(rows):
    """Scales of v from 2^-40 to 2^10 within one prefix: weights carry them relative to the largest yet.
    30 sequences: the tensor memory path, 4: the other."""
    rng = np.random.default_rng(6)
    ref = R.Cache(1, 40, 16, 1, 128, "e4m3")
    size = np.exp2(rng.integers(-30, 2, (1, 2, 40, 16, 1, 1)).astype(float))
    size[:, 0] = 1.0
    ref.values, ref.bytes = R.quantise((rng.standard_normal(ref.values.shape) * size).astype(np.float32))
    small = R.Cache(1, 40, 16, 1, 128, "e4m3")
    size[:, 1] = 2.0 ** -24
    small.values, small.bytes = R.quantise((rng.standard_normal(ref.values.shape) * size).astype(np.float32))
    for cache in (ref, small):
        c, _, _ = device_cache(cache)
        pt = np.arange(40, dtype=np.int32)
        q = torch.from_numpy(rng.standard_normal((rows, 1, 2, 128))).to(torch.float16).cuda()
        # f16 outputs below its normal range are off by up to half its smallest step
        n, t, hq, hd = q.shape
        out = torch.empty_like(q)
        work = torch.empty(c.attend_workspace_bytes(n, t, hq, 0, 640), dtype=torch.uint8, device="cuda")
        c.attend(0, q, out, None, None, torch.from_numpy(pt).cuda(), 640, workspace=work)
        o, _, a, e = R.attend(cache, 0, q.double().cpu().numpy(), np.zeros((n, 0), np.int32), [0] * n, pt, 640, hd ** -0.5)
        tol = 1.05 * (2 * 2.0 ** -11 + 2 * e[..., None]) * a + 2.0 ** -25
        assert (np.abs(out.double().cpu().numpy() - o) <= tol).all()


def test_bad_blocks_and_a_nan():
    rng = np.random.default_rng(7)
    ref = filled(rng, (1, 40, 16, 2), 128, "bf16", False)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, arena, _ = device_cache(ref, status=status)
    pt = rng.permutation(40)[:30].astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((25, 1, 8, 128))).to(torch.bfloat16).cuda()
    check(ref, c, q, pt, 470, None, None, "bf16")
    assert status.item() == 0
    broken = pt.copy()
    broken[[0, 1, 2, 3, 4, 5, 6, 7, 12, 29]] = [-1, 40, 1 << 30, -7, 99, -1, -1, -1, -(1 << 31), 41]    # the whole first tile among them
    check(ref, c, q, broken, 470, None, None, "bf16")
    assert status.item() == 4
    # NaN behind the prefix's end has no influence; in it, it is loud
    want = check(ref, c, q, pt, 470, None, None, "bf16")
    values = arena.view(torch.bfloat16).view(2, 40, 16, 2, 128)
    values[:, int(pt[29]), 6:] = float("nan")
    assert torch.equal(check(ref, c, q, pt, 470, None, None, "bf16"), want)
    values[1, int(pt[3]), 5, 0, 7] = float("nan")
    out = torch.empty_like(q)
    work = torch.empty(c.attend_workspace_bytes(25, 1, 8, 0, 470), dtype=torch.uint8, device="cuda")
    c.attend(0, q, out, None, None, torch.from_numpy(pt).cuda(), 470, workspace=work)
    assert torch.isnan(out[..., :4, 7]).all() and torch.isfinite(out[..., 4:, :]).all()


def test_captured_and_repeated_calls_give_the_same_bits():
    rng = np.random.default_rng(8)
    ref = filled(rng, (1, 100, 16, 2), 128, "e4m3", False)
    c, _, _ = device_cache(ref)
    pt, table = make_tables(rng, 100, 16, 900, [20] * 12)
    q = torch.from_numpy(rng.standard_normal((12, 1, 16, 128))).to(torch.bfloat16).cuda()
    dev = [torch.from_numpy(x).cuda() for x in (table, np.full(12, 20, np.int32), pt)]
    want = check(ref, c, q, pt, 900, table, [20] * 12, "bf16")
    out = torch.empty_like(q)
    work = torch.empty(c.attend_workspace_bytes(12, 1, 16, table.shape[1], 900), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.attend(0, q, out, dev[0], dev[1], dev[2], 900, workspace=work, stream=side)
    for _ in range(5):
        out.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("kv,hkv,seqs,prefix", [("e4m3", 37, 20, 4000), ("bf16", 37, 17, 4100), ("f16", 37, 9, 3999), ("e4m3", 19, 40, 5000)])
def test_many_tiles_a_block(kv, hkv, seqs, prefix):
    """Long runs of tiles in one block (more heads than splits fill the machine), in both uses of the
    slots; the definition in 64 bits on the GPU, the tolerance as above with its bound of a score's error."""
    g = torch.Generator(device="cuda").manual_seed(prefix)
    group, hd, block = (1, 128, 16) if seqs != 40 else (8, 64, 16)
    blocks = -(-prefix // block)
    io = "f16" if kv == "f16" else "bf16"
    group = 2 if seqs == 9 else group
    x = torch.randn(2, blocks, block, hkv, hd, generator=g, device="cuda")
    scales = None
    if kv == "e4m3":
        scales = torch.randint(120, 130, x.shape[:-1], generator=g, device="cuda").to(torch.uint8)
        codes = (x * 60).to(torch.float8_e4m3fn)
        arena, values = codes.view(torch.uint8), codes.double() * torch.exp2(scales.double() - 133)[..., None]
        scales = scales - 6
    else:
        arena = x.to(TORCH[kv]).view(torch.uint8)
        values = x.to(TORCH[kv]).double()
    import paper_2510_02613_b200 as E
    c = E.KvCache(arena, n_layers=1, num_blocks=blocks, block_tokens=block, n_heads=hkv, head_dim=hd, kv_type=kv, scales=scales)
    q = torch.randn(seqs, 1, hkv * group, hd, generator=g, device="cuda").to(TORCH[io])
    pt = torch.randperm(blocks, generator=g, device="cuda").int()
    k, v = (values[i][pt.long()].reshape(-1, hkv, hd)[:prefix] for i in range(2))
    score = torch.einsum("nhgd,phd->nhgp", q[:, 0].double().view(seqs, hkv, group, hd), k) * hd ** -0.5
    p = torch.softmax(score, -1)
    o, a = torch.einsum("nhgp,phd->nhgd", p, v), torch.einsum("nhgp,phd->nhgd", p, v.abs())
    size = torch.einsum("nhgd,phd->nhgp", q[:, 0].double().abs().view(seqs, hkv, group, hd), k.abs()).amax(-1) * hd ** -0.5
    e = (hd + 8) * 2.0 ** -23 * size + (prefix + 16) * 2.0 ** -23
    tol = 1.05 * (2 * (2.0 ** -11 if io == "f16" else 2.0 ** -8) + 2 * e[..., None]) * a + 1e-30
    outs = []
    for _ in range(3):
        out = torch.empty_like(q)
        work = torch.empty(c.attend_workspace_bytes(seqs, 1, hkv * group, 0, prefix), dtype=torch.uint8, device="cuda")
        c.attend(0, q, out, None, None, pt, prefix, workspace=work)
        outs.append(out)
        assert ((out[:, 0].double().view(o.shape) - o).abs() <= tol).all()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("seqs", [30, 3])
def test_queries_of_any_size_with_e4m3(seqs):
    """Rows whose elements span 2^-100 to 2^100 (bf16), and zero rows: they are brought to f16 by a power of two each."""
    rng = np.random.default_rng(11)
    ref = filled(rng, (1, 30, 16, 1), 128, "e4m3", False)
    ref.bytes[:, 0] = 127 - 9      # keys of about one
    c, _, _ = device_cache(ref)
    size = np.exp2(rng.integers(-100, 3, (seqs, 1, 4, 1)).astype(float))
    q = rng.standard_normal((seqs, 1, 4, 128)) * size
    q[0, 0, 0] = 0
    q[1, 0, 1, 1:] *= 2.0 ** -60
    check(ref, c, torch.from_numpy(q).to(torch.bfloat16).cuda(), np.arange(30, dtype=np.int32), 470, None, None, "bf16")
    big = torch.from_numpy(rng.standard_normal((seqs, 1, 4, 128)) * 2.0 ** 100).to(torch.bfloat16).cuda()
    check(ref, c, big, np.arange(30, dtype=np.int32), 470, None, None, "bf16", scale=2.0 ** -103)


def test_two_streams_with_workspaces_of_their_own():
    rng = np.random.default_rng(12)
    ref = filled(rng, (1, 130, 16, 2), 128, "bf16", False)
    c, _, _ = device_cache(ref)
    pt, table = make_tables(rng, 130, 16, 1500, [30] * 10)
    dev = [torch.from_numpy(x).cuda() for x in (table, np.full(10, 30, np.int32), pt)]
    q = torch.from_numpy(rng.standard_normal((10, 1, 16, 128))).to(torch.bfloat16).cuda()
    want = check(ref, c, q, pt, 1500, table, [30] * 10, "bf16")
    streams, outs = [torch.cuda.Stream() for _ in range(3)], [torch.empty(20, *q.shape, dtype=q.dtype, device="cuda") for _ in range(3)]
    works = [torch.empty(c.attend_workspace_bytes(10, 1, 16, table.shape[1], 1500), dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    for i in range(20):
        for s in range(3):
            c.attend(0, q, outs[s][i], dev[0], dev[1], dev[2], 1500, workspace=works[s], stream=streams[s])
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(x, want) for x in o)
