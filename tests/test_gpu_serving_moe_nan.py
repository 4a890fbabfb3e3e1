"""emoe_moe_decode: what is not a number or infinite in weights and tokens shows exactly where the formula has it,
and nowhere else - everything else keeps its bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import serving_ref as R
from test_gpu_serving_kv import TORCH
from test_gpu_serving_moe import Experts

pytestmark = pytest.mark.gpu

D, F, EXPERTS, TOP_K = 144, 272, 7, 2


def setup(w, n, io):
    rng = np.random.default_rng(n)
    ex = Experts(rng, 1, EXPERTS, D, F, w)
    x = torch.from_numpy(rng.standard_normal((n, D))).to(TORCH[io]).cuda()
    logits = torch.from_numpy(rng.standard_normal((n, EXPERTS))).float().cuda()
    return ex, x, logits, R.route(logits.cpu().numpy(), TOP_K)[0]


def run(ex, x, logits):
    out = torch.empty(len(x), D, device="cuda")
    work = torch.empty(ex.handle.decode_workspace_bytes(len(x), TOP_K, EXPERTS), dtype=torch.uint8, device="cuda")
    ex.handle.decode(0, x, logits, TOP_K, torch.arange(EXPERTS, dtype=torch.int32, device="cuda"), out, workspace=work)
    return out.cpu().numpy()


def poke(ex, proj, slot, row, col, code):
    cols = F if proj == 2 else D
    at = (proj * EXPERTS + slot) * D * F + row * cols + col
    if ex.w == "e4m3":
        ex.arena[at] = code
    else:
        ex.arena[:6 * EXPERTS * D * F].view(TORCH[ex.w])[at] = float("nan")


TYPES = [("e4m3", "bf16"), ("e4m3", "f16"), ("bf16", "bf16"), ("f16", "f16")]
TOKENS = [1, 4, 8, 13, 16, 31, 64]


@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("w,io", TYPES)
def test_a_down_weight_that_is_not_a_number(w, io, n):
    """It makes its output NaN for the tokens that chose the expert; both NaN codes, in either half of a tile's
    rows, at the start, inside and at the end of the k axis."""
    ex, x, logits, ids = setup(w, n, io)
    want = run(ex, x, logits)
    assert np.isfinite(want).all()
    expect = np.zeros((n, D), bool)
    slots = list(dict.fromkeys(int(e) for e in ids.reshape(-1)))[:3]
    for slot, row, col, code in zip(slots, (3, 60, 143), (0, 131, F - 1), (0x7f, 0xff, 0x7f)):
        poke(ex, 2, slot, row, col, code)
        expect[(ids == slot).any(1), row] = True
    got = run(ex, x, logits)
    assert expect.any() and np.array_equal(np.isnan(got), expect)
    assert np.array_equal(got[~expect], want[~expect])


@pytest.mark.parametrize("proj", [0, 1])
@pytest.mark.parametrize("n", [1, 16, 64])
@pytest.mark.parametrize("w,io", TYPES)
def test_a_gate_or_up_weight_that_is_not_a_number(w, io, n, proj):
    """It makes a hidden value NaN, and with it every output of the tokens that chose the expert."""
    ex, x, logits, ids = setup(w, n, io)
    want = run(ex, x, logits)
    slot = int(ids[0, 0])
    poke(ex, proj, slot, F - 3, D - 1, 0xff)
    hit = (ids == slot).any(1)
    got = run(ex, x, logits)
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], want[~hit])


@pytest.mark.parametrize("n", [1, 3, 8, 16, 64])
@pytest.mark.parametrize("w,io", TYPES)
def test_tokens_that_are_not_finite(w, io, n):
    """A token with a NaN gives NaN, one with an infinity nothing finite; the tokens beside it keep their bits."""
    ex, x, logits, _ = setup(w, n, io)
    want = run(ex, x, logits)
    for value in (float("nan"), float("inf"), -float("inf")):
        y = x.clone()
        y[n // 2, D - 5] = value
        got = run(ex, y, logits)
        assert np.isnan(got[n // 2]).all() if value != value else not np.isfinite(got[n // 2]).any()
        rest = np.arange(n) != n // 2
        assert np.array_equal(got[rest], want[rest])
