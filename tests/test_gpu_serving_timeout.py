"""The bounded waits of emoe_kv_attend's tensor core path: one that runs out is reported, what it would have
computed is not a number, and the next call is right."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_serving_attend import make_tables
from test_gpu_serving_kv import device_cache
from test_gpu_serving_prefix_wide import heads_for, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,seqs", [("bf16", 12), ("bf16", 40), ("e4m3", 12), ("e4m3", 40)])
def test_expired_waits_are_reported_and_the_next_call_is_right(kv, seqs):
    """12 sequences of 8 rows a head: one row tile on alternating tiles of tokens; 40: pairs of row tiles."""
    rng = np.random.default_rng(3)
    prefix = 1900
    hkv = heads_for(8 * seqs, prefix)
    ref = wide(rng, (1, 200, 16, hkv), 128, kv)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c, _, _ = device_cache(ref, status=status)
    lens = [int(n) for n in rng.integers(1, 20, seqs)]
    pt, table = make_tables(rng, 200, 16, prefix, lens)
    dev = [torch.from_numpy(x).cuda() for x in (table, np.array(lens, np.int32), pt)]
    q = torch.from_numpy(rng.standard_normal((seqs, 1, 8 * hkv, 128)) * 0.3).to(torch.bfloat16).cuda()
    work = torch.empty(c.attend_workspace_bytes(seqs, 1, 8 * hkv, table.shape[1], prefix), dtype=torch.uint8, device="cuda")

    def call(limit):
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
        c.attend(0, q, out, dev[0], dev[1], dev[2], prefix, lse=lse, workspace=work, wait_limit_us=limit)
        torch.cuda.synchronize()
        return out, lse

    want = call(0)
    assert status.item() == 0 and torch.isfinite(want[0]).all() and torch.isfinite(want[1]).all()
    for out in call(-1):                # every wait that is not over when it is asked runs out
        assert torch.isnan(out).all()
    assert status.item() == 10
    status.zero_()
    for limit in (0, 2000000):
        for x, y in zip(want, call(limit)):
            assert torch.equal(x, y)
    assert status.item() == 0
