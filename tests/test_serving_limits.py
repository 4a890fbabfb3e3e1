"""Refusals, sizes and checks of the serving operators on the CPU, beside those of test_serving_*.py."""
from __future__ import annotations

import ctypes

import pytest

import paper_2510_02613_b200 as E
from paper_2510_02613_b200 import binding as B
from test_serving_attend import _call as attend


@pytest.mark.parametrize("change", [dict(wait_limit_us=-2), dict(wait_limit_us=-(1 << 31)), dict(reserved2=1)])
def test_attend_wait_limits(change):
    assert attend(**change) == 1
    assert attend(wait_limit_us=-1, n_seqs=0) == 0


@pytest.mark.parametrize("w", ["bf16", "e4m3"])
def test_a_layer_workspace_is_enough_for_fewer_tokens(w):
    e = E.ExpertArena(1 << 24, n_layers=1, n_slots=140, d_model=2048, d_ff=768, w_type=w)
    need = [e.decode_workspace_bytes(n, 8, 128, 1) for n in range(65)]
    assert need == sorted(need) and need[0] == 0 and need[1] > 0
    for n in (1, 7, 8, 9, 16, 17, 64):
        sizes = [e.decode_workspace_bytes(n, k, 128, s) for k, s in ((1, 0), (1, 1), (4, 1), (8, 1), (8, 24))]
        assert sizes == sorted(sizes)
    # what the call itself asks for is never more than the query said
    arena = B._ExpertArena(1 << 24, None, 0, 1, 140, 2048, 768, e.w_type, 0, 0)
    for n in range(1, 65):
        p = B._Moe(1 << 20, 1 << 21, 1 << 22, 1 << 23, None, None, 1 << 28, need[n], 2048, 128, 2048, n, 128, 1, 8, 0, 0, 1, 1.0, 0)
        for m in range(1, n + 1):
            p.n_tokens = m
            assert B.lib().emoe_moe_decode(ctypes.byref(arena), 0, ctypes.byref(p), None) == 8     # only the arena is at fault
