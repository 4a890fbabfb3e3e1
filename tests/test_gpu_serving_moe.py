"""emoe_moe_decode on the GPU against the 64-bit definition.

Tolerance of an output element, with u the half step of the 16-bit type and s = 2^-23 the step of a
truncating 32-bit adder: gate and up are off by at most d = (D + 8) s sum|w||x| each, so that a hidden
value w silu(g) u is off by |w| (1.1 |u| d_g + |silu(g)| d_u) (|silu'| <= 1.1) and by u of itself when
it is rounded; these pass through sum |Wdown|; the last sum adds (pairs F + 8) s of its magnitudes and the result is
rounded once (u, or 2^-24 for 32-bit outputs).  Second orders are covered by a factor 1.05."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import serving_ref as R
from test_gpu_serving_kv import TORCH

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def up(a, b):
    return -(-a // b) * b


class Experts:
    """Random matrices [layers][3][slots], their arena on the device, and the definition."""

    def __init__(self, rng, layers, slots, d, f, w="bf16", fused=False, stride=0, scale=1.0):
        self.d, self.f, self.w = d, f, w
        m = d * f * R.TYPE_BYTES[w]
        raw = rng.standard_normal((layers, 3, slots, d * f)) * scale / np.sqrt(d)
        if w == "e4m3":
            codes = torch.from_numpy(np.clip(raw * np.sqrt(d) * 100, -440, 440)).float().to(torch.float8_e4m3fn)
            blocks = up(d, 128) // 128 * (up(f, 128) // 128)
            scales = torch.from_numpy(rng.uniform(0.5, 1.5, (layers, 3, slots, blocks)) * scale / 100 / np.sqrt(d)).float()
            head = codes.view(torch.uint8).reshape(-1)
            arena = torch.zeros(up(head.numel(), 256) + scales.numel() * 4, dtype=torch.uint8)
            arena[:head.numel()] = head
            arena[up(head.numel(), 256):] = scales.view(torch.uint8).reshape(-1)
            values = codes.double().numpy()
        else:
            t = torch.from_numpy(raw).to(TORCH[w])
            values = t.double().numpy()
            if fused:
                arena = torch.cat([torch.cat([torch.stack([t[l, 0], t[l, 1]], 1).reshape(-1), t[l, 2].reshape(-1)]) for l in range(layers)]).view(torch.uint8)
            else:
                arena = t.view(torch.uint8).reshape(layers, 3, slots, m)
                if stride:
                    arena = torch.nn.functional.pad(arena, (0, stride - m), value=0xff)
                arena = arena.reshape(-1)
        self.mats = []
        for l in range(layers):
            row = []
            for p in range(3):
                rows, cols = (d, f) if p == 2 else (f, d)
                v = values[l, p].reshape(slots, rows, cols)
                if w == "e4m3":
                    s = scales[l, p].double().numpy().reshape(slots, up(rows, 128) // 128, up(cols, 128) // 128)
                    v = v * s[:, np.arange(rows) // 128][:, :, np.arange(cols) // 128]
                row.append(v)
            self.mats.append(row)
        self.arena = arena.cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.handle = E.ExpertArena(self.arena, n_layers=layers, n_slots=slots, d_model=d, d_ff=f, w_type=w, fused_w13=fused,
                                    matrix_stride=stride, status=self.status)

    def reference(self, layer, x, ids, weights, table, n_shared, n_experts, u):
        """(y, tolerance before the last rounding)"""
        s = 2.0 ** -23
        y, tol = np.zeros((len(x), self.d)), np.zeros((len(x), self.d))
        gate, upm, down = self.mats[layer]
        for t in range(len(x)):
            pairs = [(int(e), w) for e, w in zip(ids[t], weights[t]) if e >= 0] + [(n_experts + i, 1.0) for i in range(n_shared)]
            pairs = [(table[e], w) for e, w in pairs if 0 <= table[e] < len(gate)]
            size = np.zeros(self.d)
            for slot, w in pairs:
                g, v = gate[slot] @ x[t], upm[slot] @ x[t]
                dg, dv = ((self.d + 8) * s * (np.abs(m[slot]) @ np.abs(x[t])) for m in (gate, upm))
                with np.errstate(over="ignore"):
                    silu = g / (1 + np.exp(-g))
                h = w * silu * v
                y[t] += down[slot] @ h
                a = np.abs(down[slot])
                tol[t] += a @ (np.abs(w) * (1.1 * np.abs(v) * dg + np.abs(silu) * dv) + (u + 8 * s) * np.abs(h))
                size += a @ np.abs(h)
            tol[t] += (len(pairs) * self.f + 8) * s * size
        return y, tol


def check(ex, x, logits, k, table, n_shared=0, layer=0, renormalize=True, routed_scale=1.0, out_type=None, io="bf16", stream=None, out=None):
    n = len(x)
    out_type = out_type or io
    out = torch.full((n, ex.d), 3.0, dtype=TORCH[out_type], device="cuda") if out is None else out
    ids = torch.full((n, k), -7, dtype=torch.int32, device="cuda")
    weights = torch.full((n, k), -7.0, device="cuda")
    work = torch.full((ex.handle.decode_workspace_bytes(n, k, logits.shape[1], n_shared),), 0xff, dtype=torch.uint8, device="cuda")
    ex.handle.decode(layer, x, logits, k, torch.from_numpy(np.asarray(table, np.int32)).cuda(), out, n_shared=n_shared,
                     renormalize=renormalize, routed_scale=routed_scale, ids_out=ids, weights_out=weights, workspace=work, stream=stream)
    torch.cuda.synchronize()
    want_ids, p = R.route(logits.cpu().numpy(), k)
    if renormalize:
        total = p.sum(1, keepdims=True)
        p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
    p = p * routed_scale
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    # exp is off by at most 2 ulp of 32 bits and its argument by half an ulp of at most 100; sum, quotient, product
    assert np.abs(weights.double().cpu().numpy() - p).max() <= 1e-5 * abs(routed_scale)
    y, tol = ex.reference(layer, x.double().cpu().numpy(), want_ids, weights.double().cpu().numpy(), table, n_shared, logits.shape[1], HALF_STEP[io])
    tol = 1.05 * (tol + HALF_STEP[out_type] * (np.abs(y) + tol)) + 1e-30
    off = np.abs(out.double().cpu().numpy() - y) / tol
    assert (off <= 1).all(), "%.3g times the tolerance at %s" % (np.nanmax(off), np.unravel_index(np.nanargmax(off), off.shape))
    return out


CASES = [
    # w, io, fused, tokens, d, f, experts, k, shared
    ("bf16", "bf16", False, 1, 64, 32, 4, 1, 0),
    ("bf16", "bf16", False, 1, 256, 176, 60, 6, 2),
    ("bf16", "bf16", True, 5, 272, 48, 8, 2, 0),
    ("f16", "f16", False, 9, 112, 64, 33, 4, 1),
    ("f16", "f16", True, 17, 16, 16, 5, 5, 0),            # a single block of k that no lane fills
    ("bf16", "bf16", False, 33, 336, 208, 16, 3, 1),
    ("bf16", "bf16", True, 64, 512, 96, 128, 8, 0),
    ("e4m3", "bf16", False, 1, 256, 128, 8, 2, 1),
    ("e4m3", "f16", False, 3, 400, 272, 12, 4, 0),        # blocks of 128 that end inside
    ("e4m3", "bf16", False, 16, 144, 160, 40, 6, 2),
    ("e4m3", "bf16", False, 64, 384, 48, 20, 2, 0),
    ("e4m3", "f16", False, 30, 16, 400, 3, 3, 1),
    ("bf16", "bf16", False, 8, 1024, 512, 300, 16, 0),    # more than 256 experts, a longer k axis
]


@pytest.mark.parametrize("w,io,fused,n,d,f,experts,k,shared", CASES)
def test_layer(w, io, fused, n, d, f, experts, k, shared):
    rng = np.random.default_rng(n * 7 + d)
    ex = Experts(rng, 2, experts + shared, d, f, w, fused)
    x = torch.from_numpy(rng.standard_normal((n, d))).to(TORCH[io]).cuda()
    logits = torch.from_numpy(rng.standard_normal((n, experts))).float().cuda()
    table = np.concatenate([rng.permutation(experts), experts + np.arange(shared)])
    check(ex, x, logits, k, table, shared, layer=1, io=io)
    check(ex, x, logits, k, table, shared, layer=0, io=io, renormalize=False, routed_scale=2.5, out_type="f32")


def test_ranks_of_an_expert_parallel_group_add_up():
    """Experts of other ranks are left out; the ranks' 32-bit outputs add up to the whole layer."""
    rng = np.random.default_rng(3)
    whole = Experts(rng, 1, 12, 128, 64)
    x = torch.from_numpy(rng.standard_normal((6, 128))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.standard_normal((6, 12))).float().cuda()
    total = 0
    for part in (range(0, 5), range(5, 6), range(6, 12)):
        table = np.array([e if e in part else -1 for e in range(12)])
        total = total + check(whole, x, logits, 4, table, out_type="f32").double()
    one = check(whole, x, logits, 4, np.arange(12), out_type="f32").double()
    assert (total - one).abs().max().item() <= 12 * 2.0 ** -23 * 64 * one.abs().max().item()
    nothing = check(whole, x, logits, 4, np.full(12, -1))
    assert not nothing.any()


def test_logits_where_the_choice_can_go_wrong():
    """Equal logits, minus infinity, NaN, fewer choices than top_k, large ones, negative zero."""
    inf, nan = float("inf"), float("nan")
    rows = [[1.0] * 7, [-inf] * 7, [nan] * 7, [-inf, 2, -inf, -inf, nan, 2, -inf], [88, -88, 90, 89.99, 0, 0, 0],
            [0.0, -0.0, 0, -0.0, -1, -2, -3], [-300, -301, -302, -303, -304, -305, -306], [3e38, -3e38, 1, 0, 0, 0, 0]]
    rng = np.random.default_rng(4)
    ex = Experts(rng, 1, 8, 64, 32)
    x = torch.from_numpy(rng.standard_normal((len(rows), 64))).to(torch.bfloat16).cuda()
    logits = torch.tensor(rows, device="cuda")
    logits[5] = torch.where(logits[5] == 0, 0.0, logits[5])    # which zero comes first is not the definition's matter
    for renormalize in (True, False):
        for k in (1, 3, 7):
            out = check(ex, x, logits, k, np.arange(8), 1, renormalize=renormalize)
    assert torch.isfinite(out).all()


def test_slots_beyond_the_arena_are_left_out_and_reported():
    rng = np.random.default_rng(5)
    ex = Experts(rng, 1, 4, 64, 32)
    x = torch.from_numpy(rng.standard_normal((3, 64))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.standard_normal((3, 6))).float().cuda()
    check(ex, x, logits, 3, [0, 1, 2, 3, -1, -9])
    assert ex.status.item() == 0
    check(ex, x, logits, 6, [0, 1, 4, 3, 1 << 30, 2])
    assert ex.status.item() == 3


def test_slab_strides_and_strided_rows():
    rng = np.random.default_rng(6)
    ex = Experts(rng, 2, 5, 96, 48, stride=1 << 14)
    wide = torch.from_numpy(rng.standard_normal((4, 200))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.standard_normal((4, 11))).float().cuda()
    target = torch.full((4, 100), 9.0, dtype=torch.bfloat16, device="cuda")
    check(ex, wide[:, 8:104], logits[:, 3:8], 2, np.arange(5), layer=1, out=target[:, 2:98])
    assert bool((target[:, :2] == 9).all()) and bool((target[:, 98:] == 9).all())


def test_hidden_values_beyond_f16():
    """silu(gate) * up beyond 65504 stands as 65504: finite, and of the right sign."""
    rng = np.random.default_rng(7)
    ex = Experts(rng, 1, 2, 64, 32, "f16", scale=400.0)
    x = torch.full((1, 64), 2.0, dtype=torch.float16, device="cuda")
    out = torch.empty(1, 64, device="cuda")
    work = torch.empty(ex.handle.decode_workspace_bytes(1, 2, 2), dtype=torch.uint8, device="cuda")
    ex.handle.decode(0, x, torch.zeros(1, 2, device="cuda"), 2, torch.arange(2, dtype=torch.int32, device="cuda"), out, workspace=work)
    assert torch.isfinite(out).all()


def test_captured_call_follows_the_router():
    rng = np.random.default_rng(8)
    ex = Experts(rng, 1, 20, 128, 64, "e4m3")
    x = torch.from_numpy(rng.standard_normal((12, 128))).to(torch.bfloat16).cuda()
    logits = torch.zeros(12, 20, device="cuda")
    table = torch.arange(20, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    work = torch.empty(ex.handle.decode_workspace_bytes(12, 4, 20), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ex.handle.decode(0, x, logits, 4, table, out, workspace=work, stream=side)
    for _ in range(3):
        logits.normal_()
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        assert torch.equal(check(ex, x, logits, 4, np.arange(20)), first)     # the same bits outside the graph


def test_repeated_calls_give_the_same_bits():
    rng = np.random.default_rng(9)
    ex = Experts(rng, 1, 40, 512, 256)
    x = torch.from_numpy(rng.standard_normal((40, 512))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.standard_normal((40, 40))).float().cuda()
    table = torch.arange(40, dtype=torch.int32, device="cuda")
    outs = torch.empty(20, 40, 512, dtype=torch.bfloat16, device="cuda")
    works = [torch.empty(ex.handle.decode_workspace_bytes(40, 6, 40), dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        ex.handle.decode(0, x, logits, 6, table, outs[i], workspace=works[i % 2], stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, outs[0]) for o in outs)


@pytest.mark.parametrize("w,io", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("n", [7, 15, 16, 31, 64])
def test_experts_with_few_and_with_all_tokens(w, io, n):
    """Column tiles: experts that 0, 1, 8, 9, 17, 33 and all tokens chose, and shared ones, in one call."""
    rng = np.random.default_rng(n)
    ex = Experts(rng, 1, 9, 400, 208, w)
    x = torch.from_numpy(rng.standard_normal((n, 400))).to(TORCH[io]).cuda()
    logits = torch.full((n, 7), -float("inf"))
    for e, count in enumerate((0, 1, 8, 9, 17, 33, 64)):
        logits[torch.from_numpy(rng.permutation(n)[:count]), e] = float(e)
    check(ex, x, logits.cuda(), 4, np.concatenate([rng.permutation(7), [7, 8]]), 2, io=io)


@pytest.mark.parametrize("d", [2368, 2384, 4752, 7120])
@pytest.mark.parametrize("w,n", [("bf16", 2), ("bf16", 12), ("bf16", 64), ("e4m3", 3), ("e4m3", 13), ("e4m3", 40)])
def test_outputs_of_every_width(d, w, n):
    """Widths at which the rows of an output take one block an SM, up to two, up to three and more."""
    rng = np.random.default_rng(d + n)
    ex = Experts(rng, 1, 7, d, 80, w)
    x = torch.from_numpy(rng.standard_normal((n, d))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.standard_normal((n, 6))).float().cuda()
    check(ex, x, logits, 2, np.arange(7), 1)


@pytest.mark.parametrize("experts", [300, 1024])
def test_the_most_choices(experts):
    """64 tokens with 32 choices each, with tables that leave room for the wider blocks and that do not."""
    rng = np.random.default_rng(experts)
    ex = Experts(rng, 1, experts, 64, 16)
    x = torch.from_numpy(rng.standard_normal((64, 64))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.standard_normal((64, experts))).float().cuda()
    check(ex, x, logits, 32, rng.permutation(experts))


def test_one_slot_for_two_experts_is_reported():
    """A table that names a slot twice: reported when a token chooses both, other tokens keep their results."""
    rng = np.random.default_rng(9)
    ex = Experts(rng, 1, 3, 64, 32)
    x = torch.from_numpy(rng.standard_normal((2, 64))).to(torch.bfloat16).cuda()
    logits = torch.tensor([[9.0, 8, 0, 1], [0.0, 1, 9, 8]], device="cuda")
    want = check(ex, x[1:], logits[1:], 2, np.array([0, -1, 1, 2]))
    table, out = torch.tensor([0, 1, 1, 2], dtype=torch.int32, device="cuda"), torch.zeros_like(x)
    work = torch.empty(ex.handle.decode_workspace_bytes(2, 2, 4), dtype=torch.uint8, device="cuda")
    ex.handle.decode(0, x, logits, 2, table, out, workspace=work)
    assert ex.status.item() == 0 and torch.equal(out[1:], want)
    logits[0] = torch.tensor([0.0, 9, 8, 1])
    ex.handle.decode(0, x, logits, 2, table, out, workspace=work)
    assert ex.status.item() == 3 and torch.equal(out[1:], want)


@pytest.mark.parametrize("w", ["bf16", "e4m3"])
def test_an_arena_longer_than_32_bit_offsets(w):
    """The last of 2048 slots in the second of two layers, more than 2^32 bytes from the arena's start."""
    rng = np.random.default_rng(10)
    d, f = (512, 512) if w == "bf16" else (1024, 768)
    ex = Experts(rng, 1, 4, d, f, w)
    x = torch.from_numpy(rng.standard_normal((9, d))).to(torch.bfloat16).cuda()
    logits = torch.from_numpy(rng.standard_normal((9, 4))).float().cuda()
    table = rng.permutation(4)
    want = check(ex, x, logits, 2, table)
    m = d * f * (2 if w == "bf16" else 1)
    small = ex.arena.flatten().view(torch.uint8)
    weights = 2 * 3 * 2048 * m
    scales = 2 * 3 * 2048 * (d // 128) * (f // 128) * 4 if w == "e4m3" else 0
    big = torch.empty(weights + scales, dtype=torch.uint8, device="cuda")
    big[:weights].view(2, 3, 2048, m)[1, :, -4:] = small[:12 * m].view(3, 4, m)
    if scales:
        big[weights:].view(2, 3, 2048, -1)[1, :, -4:] = small[12 * m:].view(3, 4, -1)
    handle = E.ExpertArena(big, n_layers=2, n_slots=2048, d_model=d, d_ff=f, w_type=w)
    out = torch.empty_like(want)
    work = torch.empty(handle.decode_workspace_bytes(9, 2, 4), dtype=torch.uint8, device="cuda")
    handle.decode(1, x, logits, 2, torch.from_numpy((table + 2044).astype(np.int32)).cuda(), out, workspace=work)
    assert torch.equal(out, want)
