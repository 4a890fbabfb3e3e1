"""Handles on arenas that are given as device addresses: the same bits as with tensors, CPU tensors refused."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
from test_gpu_serving_kv import device_cache, filled

pytestmark = pytest.mark.gpu


def test_cache_and_experts_by_address():
    rng = np.random.default_rng(1)
    ref = filled(rng, (1, 12, 16, 2), 64, "e4m3", False)
    by_tensor, arena, scales = device_cache(ref)
    by_address = E.KvCache(arena.data_ptr(), n_layers=1, num_blocks=12, block_tokens=16, n_heads=2, head_dim=64, kv_type="e4m3", scales=scales.data_ptr())
    table = torch.from_numpy(rng.permutation(12).astype(np.int32).reshape(3, 4)).cuda()
    lens = torch.tensor([64, 3, 40], dtype=torch.int32, device="cuda")
    q = torch.randn(3, 1, 4, 64, device="cuda", dtype=torch.bfloat16)
    k = torch.randn(5, 2, 64, device="cuda", dtype=torch.bfloat16)
    slots = torch.tensor([3, 77, -1, 100, 20], device="cuda")
    work = torch.empty(by_tensor.attend_workspace_bytes(3, 1, 4, 4), dtype=torch.uint8, device="cuda")
    outs = []
    for c in (by_tensor, by_address):
        c.append(0, k, -k, slots)
        back = [torch.zeros_like(k) for _ in range(2)]
        c.gather(0, slots, *back)
        out = torch.empty_like(q)
        c.attend(0, q, out, table, lens, workspace=work)
        outs.append([out] + back)
    assert all(torch.equal(x, y) for x, y in zip(*outs)) and outs[0][1][0].any()
    with pytest.raises(ValueError, match="cpu"):
        by_address.attend(0, q, torch.empty_like(q), table, lens.cpu(), workspace=work)
    for c in (by_tensor, by_address):
        with pytest.raises(ValueError, match="workspace"):
            c.attend(0, q, torch.empty_like(q), table, lens, workspace=work.cpu())

    weights = (torch.randn(3 * 4 * 64 * 32, device="cuda") * 0.1).bfloat16()
    x, logits = torch.randn(3, 64, device="cuda", dtype=torch.bfloat16), torch.randn(3, 4, device="cuda")
    slot_of = torch.arange(4, dtype=torch.int32, device="cuda")
    ys = []
    for a in (weights.view(torch.uint8), weights.data_ptr()):
        e = E.ExpertArena(a, n_layers=1, n_slots=4, d_model=64, d_ff=32)
        y = torch.empty_like(x)
        space = torch.empty(e.decode_workspace_bytes(3, 2, 4), dtype=torch.uint8, device="cuda")
        e.decode(0, x, logits, 2, slot_of, y, workspace=space)
        with pytest.raises(ValueError, match="workspace"):
            e.decode(0, x, logits, 2, slot_of, y, workspace=space.cpu())
        ys.append(y)
    assert torch.equal(*ys) and ys[0].any()
