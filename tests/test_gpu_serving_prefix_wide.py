"""emoe_kv_attend where rows times prefix are many enough (16-row tiles x tokens x KV heads from 2^17 on) for the
5th-generation tensor core path: the shapes and the values of test_gpu_serving_prefix with more heads,
against the same 64-bit definition computed on the GPU, with the tolerance of test_gpu_serving_attend."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import serving_ref as R
from test_gpu_serving_attend import HALF_STEP, check, make_tables
from test_gpu_serving_kv import TORCH, device_cache, filled

pytestmark = pytest.mark.gpu


def definition(cache, layer, q, table, own_lens, prefix_table, prefix_len, scale):
    """serving_ref.attend, vectorised on the GPU in 64 bits."""
    n, t, hq, hd = q.shape
    blocks, block, heads = cache.dims[2], cache.dims[3], cache.dims[4]
    kv = torch.from_numpy(cache.values[layer]).cuda()
    if cache.kv_type == "e4m3":
        kv = kv * torch.from_numpy(R.scale_value(cache.bytes[layer])).cuda()[..., None]
    kv = kv.reshape(2, blocks * block, heads, hd)

    def tokens(ids, count):
        """Slots of the first `count` tokens of each row of ids, and which of them lie in the pool."""
        ids = torch.from_numpy(np.ascontiguousarray(ids)).cuda().long()
        j = torch.arange(count, device="cuda")
        b = ids[..., j // block]
        return b.clamp(0, blocks - 1) * block + j % block, (b >= 0) & (b < blocks)

    qg = torch.from_numpy(q).cuda().view(n, t, heads, hq // heads, hd)
    k_abs = lambda eq, k: torch.einsum(eq, qg.abs(), k.abs()) * abs(scale)    # noqa: E731
    pt, fine = tokens(prefix_table if prefix_len else np.zeros(1, np.int32), prefix_len)
    pk, pv = kv[0][pt], kv[1][pt]
    low = torch.tensor(-float("inf"), dtype=torch.float64, device="cuda")
    scores, sizes = [torch.where(fine, torch.einsum("nthgd,phd->nthgp", qg, pk) * scale, low)], [torch.where(fine, k_abs("nthgd,phd->nthgp", pk), 0)]
    width = max(own_lens) if len(own_lens) else 0
    if width:
        own, inside = tokens(table, width)
        ok, ov = kv[0][own], kv[1][own]
        lens = torch.tensor(own_lens, device="cuda")[:, None, None] - t + 1 + torch.arange(t, device="cuda")[None, :, None]
        seen = ((torch.arange(width, device="cuda") < lens) & inside[:, None])[:, :, None, None]
        scores.append(torch.where(seen, torch.einsum("nthgd,nphd->nthgp", qg, ok) * scale, low))
        sizes.append(torch.where(seen, k_abs("nthgd,nphd->nthgp", ok), 0))
    s = torch.cat(scores, -1)
    top = s.amax(-1, keepdim=True)
    w = torch.where(top > low, torch.exp(s - torch.where(top > low, top, 0)), 0)
    total = w.sum(-1, keepdim=True)
    p = torch.where(total > 0, w / total, 0)
    o, a = (torch.einsum("nthgp,phd->nthgd", p[..., :prefix_len], f(pv)) for f in (lambda x: x, torch.abs))
    if width:
        o += torch.einsum("nthgp,nphd->nthgd", p[..., prefix_len:], ov)
        a += torch.einsum("nthgp,nphd->nthgd", p[..., prefix_len:], ov.abs())
    count = (s > low).sum(-1)
    err = torch.where(count > 0, (hd + 8) * 2.0 ** -23 * torch.cat(sizes, -1).amax(-1) + (count + 16) * 2.0 ** -23, 0)
    lse = (top + torch.log(total))[..., 0]
    shape = lambda x: x.reshape(n, t, hq, *x.shape[4:]).cpu().numpy()    # noqa: E731
    return shape(o), shape(lse), shape(a), shape(err)


@pytest.fixture
def fast(monkeypatch):
    monkeypatch.setattr(R, "attend", definition)


def wide(rng, dims, hd, kv, head_major=False):
    """`filled` without its loop over vectors: random codes and scales."""
    if kv != "e4m3":
        return filled(rng, dims, hd, kv, head_major)
    ref = R.Cache(*dims, hd, kv, head_major)
    codes = rng.integers(0, 127, ref.values.shape, dtype=np.uint8) | (rng.integers(0, 2, ref.values.shape, dtype=np.uint8) << 7)
    ref.values = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    ref.bytes = rng.integers(118, 123, ref.dims).astype(np.uint8)
    return ref


def heads_for(rows, prefix):
    """KV heads that make the prefix work for the tensor core path."""
    return -(-(1 << 17) // (-(-rows // 16) * prefix))


def check_codes(ref, c, q, pt, prefix, io, scale=None):
    """check(), prefix only, for e4m3 codes that hold zeros.  Weights are f16 there, relative to the largest scale of v
    and at least 2^6 times the softmax's (the largest of which is 1 or more before the division by their sum): one that
    falls below f16's normal range is off by up to half its smallest step, 2^-25, which is 2^-31 of v's largest
    scale times the code - no part of sum p|v| where the tokens that matter have a zero in that column.  An f16
    output has the same half step, 2^-25."""
    n, t, hq, hd = q.shape
    scale = hd ** -0.5 if scale is None else scale
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    work = torch.empty(c.attend_workspace_bytes(n, t, hq, 0, prefix), dtype=torch.uint8, device="cuda")
    c.attend(0, q, out, None, None, torch.from_numpy(np.ascontiguousarray(pt)).cuda(), prefix, scale=scale, lse=lse, workspace=work)
    o, want_l, a, e = definition(ref, 0, q.double().cpu().numpy(), np.zeros((n, 0), np.int32), [0] * n, pt, prefix, scale)
    heads = ref.dims[4]
    v = np.abs(ref.values[0, 1][pt].reshape(-1, heads, hd)[:prefix]).sum(0)                          # [heads, hd]
    top = R.scale_value(ref.bytes[0, 1][pt].reshape(-1, heads)[:prefix].max(0))                      # [heads]
    floor = np.repeat(2.0 ** -31 * top[:, None] * v, hq // heads, 0) + (2.0 ** -25 if io == "f16" else 0)
    tol = 1.05 * (2 * HALF_STEP[io] + 2 * e[..., None]) * a + floor
    off = np.abs(out.double().cpu().numpy() - o) / tol
    assert (off <= 1).all(), "%.3g times the tolerance" % np.nanmax(off)
    assert (np.abs(lse.double().cpu().numpy() - want_l) <= e + 2.0 ** -21 * np.abs(want_l) + 2.0 ** -20).all()


def test_the_definition_is_the_same():
    rng = np.random.default_rng(1)
    for kv in ("bf16", "e4m3"):
        ref = wide(rng, (1, 30, 5, 2), 32, kv)
        pt, table = make_tables(rng, 30, 5, 43, [0, 3, 17, 8])
        pt[2], table[2, 1] = -1, 30
        q = rng.standard_normal((4, 3, 6, 32))
        for prefix, lens in ((43, [0, 3, 17, 8]), (0, [0, 3, 17, 8]), (43, [0] * 4)):
            want, got = (f(ref, 0, q, table, lens, pt, prefix, 0.2) for f in (R.attend, definition))
            for x, y in zip(want, got):
                assert np.array_equal(np.isinf(x), np.isinf(y))
                assert np.allclose(x[np.isfinite(x)], y[np.isfinite(x)], rtol=1e-12, atol=1e-13)


CASES = [
    # kv, io, hm, block, group, hd, q_len, prefix, sequences
    ("bf16", "bf16", False, 16, 8, 128, 1, 128, 3),       # one tile: the second slot has none
    ("bf16", "bf16", False, 16, 1, 128, 1, 129, 17),      # two tiles, one row above the small path
    ("bf16", "bf16", True, 16, 4, 128, 1, 700, 32),       # 128 rows, odd number of tiles
    ("f16", "f16", False, 5, 3, 64, 1, 333, 20),          # blocks of 5
    ("f16", "f16", True, 1, 16, 64, 2, 260, 5),           # 160 rows: two row tiles
    ("bf16", "bf16", False, 24, 8, 128, 1, 1000, 32),     # exactly 256 rows
    ("bf16", "bf16", False, 16, 8, 64, 3, 513, 13),       # 312 rows: a second block with one row tile
    ("f16", "f16", False, 16, 8, 128, 1, 2000, 70),       # 560 rows, several splits
    ("bf16", "bf16", False, 16, 8, 64, 1, 7001, 64),      # 512 rows, many splits
    ("e4m3", "bf16", False, 16, 1, 128, 1, 1111, 33),
    ("e4m3", "bf16", True, 7, 8, 64, 1, 300, 20),
    ("e4m3", "f16", False, 16, 8, 128, 2, 400, 17),
    ("e4m3", "f16", True, 16, 2, 64, 1, 129, 40),
    ("e4m3", "bf16", False, 16, 8, 128, 1, 9000, 30),
    ("bf16", "bf16", False, 16, 8, 64, 1, 9, 70),         # a prefix of nine tokens
    ("e4m3", "bf16", False, 16, 4, 128, 1, 31, 80),
]


@pytest.mark.parametrize("kv,io,hm,block,group,hd,t,prefix,seqs", CASES)
@pytest.mark.parametrize("own", [True, False])
def test_prefix(fast, kv, io, hm, block, group, hd, t, prefix, seqs, own):
    rng = np.random.default_rng(hd + prefix + seqs)
    hkv = heads_for(seqs * t * group, prefix)
    lens = [int(x) for x in rng.integers(0, 20, seqs)] if own else [0] * seqs
    pool = -(-prefix // block) + sum(-(-n // block) for n in lens) + 2
    ref = wide(rng, (1, pool, block, hkv), hd, kv, hm)
    c, arena, scales = device_cache(ref)
    pt, table = make_tables(rng, pool, block, prefix, lens)
    q = torch.from_numpy(rng.standard_normal((seqs, t, hkv * group, hd)) * (2 if kv != "e4m3" else 0.2)).to(TORCH[io]).cuda()
    if own:
        check(ref, c, q, pt, prefix, table, lens, io)
    else:
        check(ref, c, q, pt, prefix, None, None, io)


@pytest.mark.parametrize("kv,io", [("bf16", "bf16"), ("e4m3", "f16"), ("e4m3", "bf16")])
def test_scores_that_raise_the_maximum_and_signs(fast, kv, io):
    """Keys that grow along the prefix (the maximum is raised again and again), shrinking ones, a negative,
    a zero and a tiny scale."""
    rng = np.random.default_rng(5)
    hkv = heads_for(160, 795)
    ref = wide(rng, (1, 50, 16, hkv), 64, kv)
    grow = np.linspace(0.05, 6, 800).reshape(50, 16)[None, None, :, :, None] ** 2
    if kv == "e4m3":
        ref.bytes = (122 + np.floor(np.log2(grow))).astype(np.uint8) + np.zeros_like(ref.bytes)
    else:
        ref.values = torch.from_numpy(ref.values * grow[..., None]).to(TORCH[kv]).double().numpy()
    c, _, _ = device_cache(ref)
    for order in (np.arange(50), np.arange(50)[::-1]):
        pt = order.astype(np.int32)
        q = torch.from_numpy(rng.standard_normal((40, 1, 4 * hkv, 64)) * (0.2 if kv == "e4m3" else 1)).to(TORCH[io]).cuda()
        for scale in (0.125, -1.0, 0.0, 2.0 ** -30):
            if kv == "e4m3":
                check_codes(ref, c, q, pt, 795, io, scale)
            else:
                check(ref, c, q, pt, 795, None, None, io, scale=scale)


def test_small_and_large_values_in_e4m3_with_f16():
    """Scales of v from 2^-39 to 2^-7 within one prefix: weights carry them relative to the largest yet."""
    rng = np.random.default_rng(6)
    hkv = heads_for(60, 640)
    ref, small = (wide(rng, (1, 40, 16, hkv), 128, "e4m3") for _ in range(2))
    ref.bytes[:, 1] = rng.integers(127 - 39, 127 - 7, ref.bytes[:, 1].shape)
    small.bytes[:, 1] = 127 - 33
    for cache in (ref, small):
        c, _, _ = device_cache(cache)
        pt = np.arange(40, dtype=np.int32)
        q = torch.from_numpy(rng.standard_normal((30, 1, 2 * hkv, 128)) * 0.2).to(torch.float16).cuda()
        # f16 outputs below its normal range are off by up to half its smallest step
        n, t, hq, hd = q.shape
        out = torch.empty_like(q)
        work = torch.empty(c.attend_workspace_bytes(n, t, hq, 0, 640), dtype=torch.uint8, device="cuda")
        c.attend(0, q, out, None, None, torch.from_numpy(pt).cuda(), 640, workspace=work)
        o, _, a, e = definition(cache, 0, q.double().cpu().numpy(), np.zeros((n, 0), np.int32), [0] * n, pt, 640, hd ** -0.5)
        tol = 1.05 * (2 * 2.0 ** -11 + 2 * e[..., None]) * a + 2.0 ** -25
        assert (np.abs(out.double().cpu().numpy() - o) <= tol).all()


def test_bad_blocks_and_a_nan(fast):
    rng = np.random.default_rng(7)
    hkv = heads_for(100, 470)
    ref = wide(rng, (1, 40, 16, hkv), 128, "bf16")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, arena, _ = device_cache(ref, status=status)
    pt = rng.permutation(40)[:30].astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((25, 1, 4 * hkv, 128))).to(torch.bfloat16).cuda()
    want = check(ref, c, q, pt, 470, None, None, "bf16")
    assert status.item() == 0
    broken = pt.copy()
    broken[[0, 1, 2, 3, 4, 5, 6, 7, 12, 29]] = [-1, 40, 1 << 30, -7, 99, -1, -1, -1, -(1 << 31), 41]    # the whole first tile among them
    check(ref, c, q, broken, 470, None, None, "bf16")
    assert status.item() == 4
    # a prefix of which nothing is left: zero, and minus infinity
    check(ref, c, q, np.full(30, -1, np.int32), 470, None, None, "bf16")
    # NaN behind the prefix's end has no influence; in it, it is loud
    values = arena.view(torch.bfloat16).view(2, 40, 16, hkv, 128)
    values[:, int(pt[29]), 6:] = float("nan")
    assert torch.equal(check(ref, c, q, pt, 470, None, None, "bf16"), want)
    values[1, int(pt[3]), 5, 0, 7] = float("nan")
    out = torch.empty_like(q)
    work = torch.empty(c.attend_workspace_bytes(25, 1, 4 * hkv, 0, 470), dtype=torch.uint8, device="cuda")
    c.attend(0, q, out, None, None, torch.from_numpy(pt).cuda(), 470, workspace=work)
    assert torch.isnan(out[..., :4, 7]).all() and torch.isfinite(out[..., 4:, :]).all()


@pytest.mark.parametrize("kv", ["e4m3", "bf16"])
def test_captured_and_concurrent_calls_give_the_same_bits(fast, kv):
    """One call captured and replayed, and three streams at once with workspaces of their own."""
    rng = np.random.default_rng(8)
    hkv, prefix, own = heads_for(96, 1500), 1500, [20] * 12
    ref = wide(rng, (1, 130, 16, hkv), 128, kv)
    c, _, _ = device_cache(ref)
    pt, table = make_tables(rng, 130, 16, prefix, own)
    q = torch.from_numpy(rng.standard_normal((12, 1, 8 * hkv, 128)) * 0.2).to(torch.bfloat16).cuda()
    dev = [torch.from_numpy(x).cuda() for x in (table, np.full(12, 20, np.int32), pt)]
    want = check(ref, c, q, pt, prefix, table, own, "bf16")
    out = torch.empty_like(q)
    size = c.attend_workspace_bytes(12, 1, 8 * hkv, table.shape[1], prefix)
    works = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    streams[0].wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        c.attend(0, q, out, dev[0], dev[1], dev[2], prefix, workspace=works[0], stream=streams[0])
    for _ in range(5):
        out.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    outs = torch.empty(3, 10, *q.shape, dtype=q.dtype, device="cuda")
    torch.cuda.synchronize()
    for i in range(10):
        for s in range(3):
            c.attend(0, q, outs[s, i], dev[0], dev[1], dev[2], prefix, workspace=works[s], stream=streams[s])
    torch.cuda.synchronize()
    assert (outs == want).all()


def test_queries_of_any_size_with_e4m3():
    """Rows whose elements span 2^-100 to 2^100 (bf16), and zero rows: they are brought to f16 by a power of two each."""
    rng = np.random.default_rng(11)
    hkv = heads_for(120, 470)
    ref = wide(rng, (1, 30, 16, hkv), 128, "e4m3")
    c, _, _ = device_cache(ref)
    size = np.exp2(rng.integers(-100, 1, (30, 1, 4 * hkv, 1)).astype(float))
    q = rng.standard_normal((30, 1, 4 * hkv, 128)) * size
    q[0, 0, 0] = 0
    q[1, 0, 1, 1:] *= 2.0 ** -60
    check_codes(ref, c, torch.from_numpy(q).to(torch.bfloat16).cuda(), np.arange(30, dtype=np.int32), 470, "bf16")
    big = torch.from_numpy(rng.standard_normal((30, 1, 4 * hkv, 128)) * 2.0 ** 100).to(torch.bfloat16).cuda()
    check_codes(ref, c, big, np.arange(30, dtype=np.int32), 470, "bf16", scale=2.0 ** -106)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_a_cache_longer_than_32_bit_offsets_and_strided_rows(fast, kv):
    """Prefix and own tokens on the last blocks of a pool of 5.2 GB (e4m3: 4.6) each for K and V; queries and outputs with gaps."""
    import paper_2510_02613_b200 as E
    rng = np.random.default_rng(13)
    size = 2 if kv == "bf16" else 1
    heads, hd, seqs, prefix, many = 16, 128, 32, 4096, 80000 if size == 2 else 140000
    lens = [int(x) for x in rng.integers(0, 30, seqs)]
    pool = prefix // 16 + sum(-(-n // 16) for n in lens) + 1
    ref = wide(rng, (1, pool, 16, heads), hd, kv)
    _, arena, scales = device_cache(ref)
    big = torch.empty(2 * many * 16 * heads * hd * size, dtype=torch.uint8, device="cuda")
    big.view(2, many, -1)[:, -pool:] = arena.view(2, pool, -1)
    big_scales = None
    if kv == "e4m3":
        big_scales = torch.full((2 * many * 16 * heads,), 255, dtype=torch.uint8, device="cuda")
        big_scales.view(2, many, -1)[:, -pool:] = scales.view(2, pool, -1)
    c = E.KvCache(big, n_layers=1, num_blocks=many, block_tokens=16, n_heads=heads, head_dim=hd, kv_type=kv, scales=big_scales)
    pt, table = make_tables(rng, pool, 16, prefix, lens)
    wide_q = torch.full((seqs, 1, heads + 1, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide_q[:, :, :heads] = torch.from_numpy(rng.standard_normal((seqs, 1, heads, hd)) * 0.2).to(torch.bfloat16).cuda()
    wide_out = torch.full((seqs, 1, heads + 2, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    q, out = wide_q[:, :, :heads], wide_out[:, :, :heads]
    lse = torch.empty(seqs, 1, heads, device="cuda")
    at = many - pool
    dev = [torch.from_numpy(x).cuda() for x in (np.where(table < 0, -1, table + at).astype(np.int32), np.asarray(lens, np.int32), (pt + at).astype(np.int32))]
    work = torch.empty(c.attend_workspace_bytes(seqs, 1, heads, table.shape[1], prefix), dtype=torch.uint8, device="cuda")
    c.attend(0, q, out, dev[0], dev[1], dev[2], prefix, lse=lse, workspace=work)
    o, want_l, a, e = definition(ref, 0, q.double().cpu().numpy(), table, lens, pt, prefix, hd ** -0.5)
    tol = 1.05 * (2 * HALF_STEP["bf16"] + 2 * e[..., None]) * a + 1e-30
    assert (np.abs(out.double().cpu().numpy() - o) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy() - want_l) <= e + 2.0 ** -21 * np.abs(want_l) + 2.0 ** -20).all()
    assert (wide_out[:, :, heads:] == 7).all()
