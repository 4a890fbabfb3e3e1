"""emoe_moe_decode on an e4m3 arena with gate and up matrices interleaved: scales stay [3][n_slots], and the bits are
those of the plain arena."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
from test_gpu_serving_moe import Experts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [2, 12, 40])
def test_interleaved_gate_and_up_in_e4m3(n, io):
    rng = np.random.default_rng(n)
    layers, slots, d, f = 2, 5, 272, 144
    plain = Experts(rng, layers, slots, d, f, "e4m3")
    fused = plain.arena.clone()
    codes = plain.arena[:layers * 3 * slots * d * f].view(layers, 3, slots, d * f)
    for l in range(layers):
        at = fused[l * 3 * slots * d * f:]
        at[:2 * slots * d * f] = codes[l, :2].transpose(0, 1).reshape(-1)     # [slot][gate, up]
    handle = E.ExpertArena(fused, n_layers=layers, n_slots=slots, d_model=d, d_ff=f, w_type="e4m3", fused_w13=True)
    x, logits = torch.randn(n, d, device="cuda").to(io), torch.randn(n, slots, device="cuda")
    table = torch.from_numpy(rng.permutation(slots).astype(np.int32)).cuda()
    outs = [torch.empty(n, d, device="cuda") for _ in range(2)]
    for h, out in zip((plain.handle, handle), outs):
        work = torch.empty(h.decode_workspace_bytes(n, 3, slots), dtype=torch.uint8, device="cuda")
        h.decode(1, x, logits, 3, table, out, workspace=work)
    assert torch.equal(*outs) and torch.isfinite(outs[0]).all() and outs[0].any()
