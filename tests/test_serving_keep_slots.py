"""emoe_kv_keep with the slots of the extend before it: its refusals, on the CPU."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_2510_02613_b200 as E
from paper_2510_02613_b200 import binding as B


def _keep(**changes):
    c = B._KvCache(1 << 24, None, None, 2, 30, 4, 2, 64, 0, 0, 0)
    p = B._Keep(*((1 << 20) + 4096 * i for i in range(6)), 3, 5, 4, 0, 1 << 22, 40, 0)
    for name, value in changes.items():
        setattr(p, name, value)
    return B.lib().emoe_kv_keep(ctypes.byref(c), ctypes.byref(p), None)


@pytest.mark.parametrize("change,code", [(dict(reserved2=1), 1), (dict(slots=None), 1), (dict(n_slots=-1), 2), (dict(slots=(1 << 22) + 4), 5)])
def test_keep_refuses_bad_slots(change, code):
    assert _keep(**change) == code


def test_python_checks_slots():
    arena = torch.zeros(2 * 2 * 30 * 4 * 2 * 64 * 2, dtype=torch.uint8)
    c = E.KvCache(arena, n_layers=2, num_blocks=30, block_tokens=4, n_heads=2, head_dim=64)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)    # noqa: E731
    for bad in (torch.zeros(9, dtype=torch.int32), torch.zeros((3, 3), dtype=torch.int64), torch.zeros(18, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError):
            c.keep(i32(3, 5), i32(3), i32(4), i32(3, 2), i32(3), i32(3), slots=bad)
