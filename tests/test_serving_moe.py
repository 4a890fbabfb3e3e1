"""Refusals and sizes of emoe_moe_decode on the CPU; the reference's routing by hand-written cases."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import serving_ref as R
import workloads as W
from paper_2510_02613_b200 import binding as B


def _call(layer=0, experts=None, **changes):
    e = B._ExpertArena(1 << 24, None, 0, 2, 6, 64, 32, 0, 0, 0)
    p = B._Moe(1 << 20, 1 << 21, 1 << 22, 1 << 23, None, None, 1 << 28, 1 << 40, 64, 8, 64, 3, 8, 1, 2, 0, 0, 1, 1.0, 0)
    for name, value in (experts or {}).items():
        setattr(e, name, value)
    for name, value in changes.items():
        setattr(p, name, value)
    return B.lib().emoe_moe_decode(ctypes.byref(e), layer, ctypes.byref(p), None)


@pytest.mark.parametrize("change,code", [
    (dict(layer=-1), 1), (dict(layer=2), 1), (dict(x=None), 1), (dict(logits=None), 1), (dict(slot_of_expert=None), 1), (dict(out=None), 1),
    (dict(workspace=None), 1), (dict(workspace_bytes=100), 1), (dict(flags=2), 1), (dict(reserved=1), 1), (dict(io_type=2), 1),
    (dict(io_type=3), 1), (dict(out_type=1), 1), (dict(out_type=3), 1), (dict(experts=dict(arena=None)), 1), (dict(experts=dict(reserved=1)), 1),
    (dict(experts=dict(layout=8)), 1), (dict(experts=dict(type=2)), 1),
    (dict(n_tokens=-1), 2), (dict(top_k=0), 2), (dict(top_k=9), 2), (dict(n_experts=0), 2), (dict(n_shared=-1), 2), (dict(x_stride=63), 2),
    (dict(out_stride=8), 2), (dict(logits_stride=7), 2), (dict(experts=dict(n_slots=0)), 2), (dict(experts=dict(d_ff=-16)), 2),
    (dict(experts=dict(n_layers=0)), 2), (dict(experts=dict(matrix_stride=4080)), 2),
    (dict(x=(1 << 20) + 8), 5), (dict(logits=2), 5), (dict(slot_of_expert=1), 5), (dict(out=3), 5), (dict(ids_out=2), 5), (dict(weights_out=1), 5),
    (dict(workspace=(1 << 28) + 128), 5), (dict(x_stride=68), 5), (dict(experts=dict(arena=(1 << 24) + 4)), 5), (dict(experts=dict(status=1)), 5),
    (dict(experts=dict(matrix_stride=4104)), 5),
    (dict(io_type=1, out_type=1), 9), (dict(experts=dict(d_model=72)), 9), (dict(experts=dict(d_ff=24)), 9),
    (dict(experts=dict(matrix_stride=8192, layout=4)), 9), (dict(experts=dict(matrix_stride=8192, type=3)), 9),
    (dict(n_tokens=65), 11), (dict(n_experts=1025, logits_stride=2000), 11), (dict(top_k=8, n_shared=25), 11), (dict(experts=dict(n_slots=4097)), 11),
])
def test_refusals(change, code):
    assert _call(**change) == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="looks at the answer without a device")
def test_without_a_device_the_call_is_refused():
    assert _call() == 8


def test_empty_and_null():
    assert _call(n_tokens=0, x=None, out=None, workspace=None) == 0
    assert B.lib().emoe_moe_decode(None, 0, None, None) == 1
    e = B._ExpertArena(1 << 24, None, 0, 2, 6, 64, 32, 0, 0, 0)
    assert B.lib().emoe_moe_decode(ctypes.byref(e), 0, None, None) == 1
    assert B.lib().emoe_moe_decode_workspace(ctypes.byref(e), 1, 2, 8, 0, None) == 1


def test_arena_sizes_are_those_of_a_plan():
    cfg = W.ParallelConfig(1, 1, [[0, 1, 2]], 1, [], np.zeros((0, 0), np.int32))
    for b, scale, kw in ((2, 0, {}), (1, 2 * 3 * 4, dict(w_type="e4m3"))):
        with E.Plan(W.Shape(2, 3, 0, 144, 272, 1, 1, 8, 16, b, scale), cfg, cfg, host_only=True) as plan:
            e = E.ExpertArena(1 << 20, n_layers=2, n_slots=3, d_model=144, d_ff=272, **kw)
            assert plan.arena_bytes(E.PHASE_EXPERTS, E.SIDE_OLD) == [e.bytes()]
    assert E.ExpertArena(1 << 20, n_layers=2, n_slots=3, d_model=144, d_ff=272, matrix_stride=1 << 21).bytes() == 18 << 21


def test_python_checks():
    e = E.ExpertArena(torch.zeros(3 * 6 * 64 * 32 * 2, dtype=torch.uint8), n_layers=1, n_slots=6, d_model=64, d_ff=32)
    x, logits, table = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(3, 8), torch.zeros(8, dtype=torch.int32)
    good = dict(x=x, logits=logits, top_k=2, slot_of_expert=table, out=x.clone())
    for bad in (dict(x=x[:, :32]), dict(x=x.double()), dict(logits=logits.half()), dict(slot_of_expert=table[:7]), dict(n_shared=1),
                dict(slot_of_expert=table.long()), dict(out=x[:2]), dict(ids_out=torch.zeros(3, 2)), dict(weights_out=torch.zeros(3, 1)),
                dict(x=torch.zeros(64, 3, dtype=torch.bfloat16).t())):
        with pytest.raises(ValueError):
            e.decode(0, **{**good, **bad})
    with pytest.raises(ValueError):
        E.ExpertArena(torch.zeros(100, dtype=torch.uint8), n_layers=1, n_slots=6, d_model=64, d_ff=32)


def test_reference_routing():
    inf = np.inf
    ids, p = R.route([[1, 3, 3, 2], [-inf, 0, -inf, np.nan], [-inf] * 4, [np.nan] * 4], 2)
    assert ids.tolist() == [[1, 2], [1, -1], [-1, -1], [-1, -1]]
    total = np.exp([1, 3, 3, 2]).sum()
    assert np.allclose(p[0], [np.exp(3) / total] * 2) and p[1].tolist() == [1, 0] and not p[2:].any()
