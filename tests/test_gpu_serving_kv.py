"""emoe_kv_append and emoe_kv_gather on the GPU against the 64-bit definition.  Tolerance: zero -
codes, scale bytes and 16-bit values are unique (one rounding, ties to even), and every byte of the
arenas that no slot names has to stay as it was."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import serving_ref as R

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


def device_cache(ref, layers_of_garbage=True, status=None):
    """(handle, arena, scales) of a reference cache."""
    values = torch.from_numpy(ref.order(ref.values)).cuda().to(torch.float32).to(TORCH[ref.kv_type])
    arena = values.view(torch.uint8)
    scales = torch.from_numpy(ref.order(ref.bytes).copy()).cuda() if ref.kv_type == "e4m3" else None
    l, _, nb, b, h = ref.dims
    c = E.KvCache(arena, n_layers=l, num_blocks=nb, block_tokens=b, n_heads=h, head_dim=ref.head_dim, kv_type=ref.kv_type,
                  scales=scales, head_major=ref.head_major, status=status)
    return c, arena, scales


def filled(rng, dims, hd, kv, head_major):
    ref = R.Cache(*((dims[0],) + dims[1:]), hd, kv, head_major)
    x = rng.standard_normal(ref.values.shape)
    if kv == "e4m3":
        ref.values, ref.bytes = R.quantise(x.astype(np.float32))
    else:
        ref.values = torch.from_numpy(x).to(TORCH[kv]).double().numpy()
    return ref


def same(arena, scales, ref):
    got = arena.view(TORCH[ref.kv_type]).double().cpu().numpy()
    assert np.array_equal(got, ref.order(ref.values), equal_nan=True)
    if scales is not None:
        assert np.array_equal(scales.cpu().numpy(), ref.order(ref.bytes))


CASES = [
    # block, heads, hd, cache, io, head_major, tokens
    (16, 4, 128, "e4m3", "bf16", False, 33), (16, 1, 128, "e4m3", "f16", True, 7), (5, 3, 96, "e4m3", "f32", True, 1),
    (1, 2, 8, "e4m3", "bf16", False, 5), (16, 2, 256, "e4m3", "f32", False, 20), (8, 5, 32, "bf16", "bf16", True, 30),
    (16, 4, 64, "f16", "f16", False, 17), (7, 2, 72, "bf16", "f32", False, 19), (16, 2, 128, "f16", "f32", True, 40),
    (32, 16, 128, "e4m3", "bf16", False, 90),
]


@pytest.mark.parametrize("block,heads,hd,kv,io,hm,n", CASES)
def test_append_then_gather(block, heads, hd, kv, io, hm, n):
    rng = np.random.default_rng(n * 131 + hd)
    blocks = -(-n // block) + 2
    ref = filled(rng, (2, blocks, block, heads), hd, kv, hm)
    c, arena, scales = device_cache(ref)
    slots = rng.permutation(blocks * block)[:n].astype(np.int64)
    skip = rng.random(n) < 0.2
    slots[skip] = -1
    # a row of a fused projection: k and v lie in one tensor with more elements a token
    wide = torch.from_numpy(rng.standard_normal((n, 3, heads, hd)) * 10.0 ** rng.integers(-6, 4, (n, 3, heads, 1))).to(TORCH[io]).cuda()
    k, v = wide[:, 1], wide[:, 2]
    c.append(1, k, v, torch.from_numpy(slots).cuda())
    torch.cuda.synchronize()
    for kv_i, x in enumerate((k, v)):
        x = x.double().cpu().numpy()
        for i, s in enumerate(slots):
            if s < 0:
                continue
            b, o = divmod(int(s), block)
            if kv == "e4m3":
                ref.values[1, kv_i, b, o], ref.bytes[1, kv_i, b, o] = R.quantise(x[i])
            else:
                ref.values[1, kv_i, b, o] = torch.from_numpy(x[i]).float().to(TORCH[kv]).double().numpy()
    same(arena, scales, ref)
    # and back, rows of skipped tokens untouched, a slot read twice
    order = np.concatenate([slots, slots[:1]])
    out = torch.full((n + 1, 2, heads, hd), 7.0, dtype=TORCH[io], device="cuda")
    c.gather(1, torch.from_numpy(order).cuda(), out[:, 0], out[:, 1])
    for i, s in enumerate(order):
        for kv_i in range(2):
            want = np.full((heads, hd), 7.0) if s < 0 else ref.read(1, kv_i, s)
            want = torch.from_numpy(want).to(TORCH[io]).double().numpy()
            assert np.array_equal(out[i, kv_i].double().cpu().numpy(), want, equal_nan=True)


def test_values_where_the_quantiser_can_go_wrong():
    """Ties, the largest code, zero, denormal, huge, infinite and NaN vectors; each alone in a head."""
    rows = np.zeros((16, 32), np.float32)
    rows[0, :4] = 448, 17, 19, -18
    rows[1, 0] = 449
    rows[2, :2] = 448 * 2.0 ** -20, 2.0 ** -40
    rows[3, 5] = 1e-42                     # a denormal of 32 bits
    rows[4, 3] = 3.4e38
    rows[5, 3] = -3.4e38
    rows[6, 31] = np.inf
    rows[7, 0] = -np.inf
    rows[8, 9] = np.nan
    rows[10] = np.float32(2.0 ** -9) * np.arange(32) / 4     # around the smallest codes
    rows[10, 0] = 448
    rows[11] = 1.75 * 2.0 ** -3
    rows[12] = np.nextafter(np.float32(1.75), np.float32(2))
    rows[13] = 2.0 ** -149
    rows[14] = -np.linspace(0, 448, 32)
    rows[15] = np.float32(2.0 ** -126)
    ref = R.Cache(1, 2, 8, 1, 32, "e4m3")
    c, arena, scales = device_cache(ref)
    x = torch.from_numpy(rows).cuda()[:, None]
    c.append(0, x, x, torch.arange(16, device="cuda"))
    for i in range(16):
        for kv in range(2):
            ref.values[0, kv, i // 8, i % 8], ref.bytes[0, kv, i // 8, i % 8] = R.quantise(rows[i][None])
    same(arena, scales, ref)
    k, v = torch.empty_like(x), torch.empty_like(x)
    c.gather(0, torch.arange(16, device="cuda"), k, v)
    # in the output's type: 3.4e38 rounds to the code of 2^128, which 32 bits do not hold
    want = torch.from_numpy(np.stack([ref.read(0, 0, i) for i in range(16)])).float().double().numpy()
    assert np.isinf(want[4:6]).sum() == 2
    assert np.array_equal(k.double().cpu().numpy(), want, equal_nan=True)
    assert np.isnan(want[6:9]).all() and torch.equal(k.nan_to_num(), v.nan_to_num())


def test_ids_beyond_the_pool_are_skipped_and_reported():
    rng = np.random.default_rng(5)
    ref = filled(rng, (1, 3, 4, 2), 16, "e4m3", False)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, arena, scales = device_cache(ref, status=status)
    x = torch.randn(4, 2, 16, device="cuda", dtype=torch.bfloat16)
    none = torch.full((4,), -1, dtype=torch.int64, device="cuda")
    c.append(0, x, x, none)
    same(arena, scales, ref)
    assert status.item() == 0
    bad = torch.tensor([12, 1 << 31, (1 << 32) + 1, (1 << 62)], device="cuda")
    c.append(0, x, x, bad)
    same(arena, scales, ref)
    assert status.item() == 4
    status.zero_()
    out = torch.full((4, 2, 16), 3.0, device="cuda")
    c.gather(0, bad, out, out.clone())
    assert status.item() == 4 and bool((out == 3).all())


def test_every_pair_of_types_and_a_large_call():
    """The path with several vectors a thread, and each conversion, against torch's own rounding."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for kv, io in (("e4m3", "bf16"), ("e4m3", "f16"), ("e4m3", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")):
        n, h, hd = 3001, 16, 128
        k, v = (torch.randn(n, h, hd, generator=g, device="cuda").to(TORCH[io]) for _ in range(2))
        size = R.TYPE_BYTES[kv]
        arena = torch.zeros(2 * 200 * 16 * h * hd * size, dtype=torch.uint8, device="cuda")
        scales = torch.zeros(2 * 200 * 16 * h, dtype=torch.uint8, device="cuda") if kv == "e4m3" else None
        c = E.KvCache(arena, n_layers=1, num_blocks=200, block_tokens=16, n_heads=h, head_dim=hd, kv_type=kv, scales=scales)
        slots = torch.randperm(3200, generator=g, device="cuda")[:n]
        c.append(0, k, v, slots)
        k2, v2 = torch.empty_like(k), torch.empty_like(v)
        c.gather(0, slots, k2, v2)
        for a, b in ((k, k2), (v, v2)):
            if kv == "e4m3":
                top = a.float().abs().amax(-1, keepdim=True)
                m, e = torch.frexp(top)
                by = torch.exp2((e - 9 + (m > 0.875)).double())
                want = ((a.double() / by).float().to(torch.float8_e4m3fn).double() * by).to(a.dtype)
            else:
                want = a.to(TORCH[kv]).to(a.dtype)
            assert torch.equal(want, b)


def test_captured_calls_and_another_stream():
    ref = R.Cache(1, 4, 16, 2, 64, "e4m3")
    c, arena, scales = device_cache(ref)
    k = torch.randn(8, 2, 64, device="cuda", dtype=torch.bfloat16)
    slots = torch.arange(8, device="cuda")
    k2, v2 = torch.empty_like(k), torch.empty_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.append(0, k, k, slots, stream=side)
        c.gather(0, slots, k2, v2, stream=side)
    for shift in (0, 20, 40):
        k.normal_()
        slots.copy_(torch.arange(8, device="cuda") + shift)
        graph.replay()
        torch.cuda.synchronize()
        x = R.quantise(k.double().cpu().numpy())
        want = x[0] * R.scale_value(x[1])[..., None]
        assert np.array_equal(k2.double().cpu().numpy(), want) and torch.equal(k2, v2)


def test_a_cache_longer_than_32_bit_offsets():
    """Element and byte offsets beyond 2^32: the last slots of a pool of 4.6 GB each for K and V."""
    nb, b, h, hd = 35000, 16, 64, 128
    arena = torch.empty(2 * nb * b * h * hd, dtype=torch.uint8, device="cuda")
    scales = torch.empty(2 * nb * b * h, dtype=torch.uint8, device="cuda")
    c = E.KvCache(arena, n_layers=1, num_blocks=nb, block_tokens=b, n_heads=h, head_dim=hd, kv_type="e4m3", scales=scales)
    slots = torch.tensor([nb * b - 1, 0, nb * b - 16, 3], device="cuda")
    k, v = (torch.randn(4, h, hd, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    c.append(0, k, v, slots)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    c.gather(0, slots, k2, v2)
    for a, got in ((k, k2), (v, v2)):
        codes, byte = R.quantise(a.double().cpu().numpy())
        assert np.array_equal(got.double().cpu().numpy(), codes * R.scale_value(byte)[..., None])
    assert torch.equal(arena.view(2, nb * b, h, hd)[0, nb * b - 1].view(torch.float8_e4m3fn).double().cpu(),
                       torch.from_numpy(R.quantise(k[0].double().cpu().numpy())[0]))
