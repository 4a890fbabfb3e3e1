"""The paged cache's geometry and the refusals of emoe_kv_append / _gather, on the CPU."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import serving_ref as R
from paper_2510_02613_b200 import binding as B

DIMS = dict(n_layers=2, num_blocks=3, block_tokens=4, n_heads=2, head_dim=16)


@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("block_tokens,heads", [(1, 1), (4, 2), (5, 3), (16, 1)])
def test_vector_index_follows_the_reshard_layout(block_tokens, heads, head_major):
    c = E.KvCache(1 << 20, n_layers=2, num_blocks=3, block_tokens=block_tokens, n_heads=heads, head_dim=8, head_major=head_major)
    index = np.arange(2 * 2 * 3 * block_tokens * heads)
    shape = (2, 2, 3) + ((heads, block_tokens) if head_major else (block_tokens, heads))
    where = index.reshape(shape)
    where = where.swapaxes(3, 4) if head_major else where
    for l in range(2):
        for kv in range(2):
            for slot in range(3 * block_tokens):
                for h in range(heads):
                    assert c.vector_index(l, kv, slot, h) == where[l, kv, slot // block_tokens, slot % block_tokens, h]
    for bad in ((2, 0, 0, 0), (-1, 0, 0, 0), (0, 2, 0, 0), (0, 0, -1, 0), (0, 0, 3 * block_tokens, 0), (0, 0, 0, heads), (0, 0, 0, -1)):
        assert c.vector_index(*bad) == -1


def test_indices_pass_32_bits():
    c = E.KvCache(1 << 20, n_layers=40, num_blocks=1 << 20, block_tokens=1024, n_heads=64, head_dim=128)
    last = (1 << 30) - 1
    assert c.vector_index(39, 1, last, 63) == 80 * (1 << 36) - 1
    assert c.bytes()[0] == 80 * (1 << 36) * 256


def test_the_arenas_are_those_of_a_plan():
    """Codes: a KV plan with elem_bytes 1; scales: one with head_dim 1."""
    import workloads as W
    bt = np.array([[0, 1]], np.int32)
    cfg = W.ParallelConfig(1, 2, [[0]], 5, [30], bt)
    for hd, pick in ((64, 0), (1, 1)):
        with E.Plan(W.Shape(3, 1, 0, 8, 8, 4, 4, hd, 16, 1), cfg, cfg, host_only=True) as plan:
            c = E.KvCache(1 << 20, n_layers=3, num_blocks=5, block_tokens=16, n_heads=2, head_dim=64, kv_type="e4m3", scales=1 << 20)
            assert plan.arena_bytes(E.PHASE_KV, E.SIDE_OLD) == [c.bytes()[pick]] * 2


def _call(fn="emoe_kv_append", cache=None, layer=0, k=1 << 20, v=1 << 21, ks=32, vs=32, io=0, slots=1 << 22, n=3, **changes):
    c = B._KvCache(1 << 24, None, None, 2, 3, 4, 2, 16, 0, 0, 0)
    for name, value in changes.items():
        setattr(c, name, value)
    p = ctypes.byref(c) if cache is None else cache
    if fn == "emoe_kv_append":
        return B.lib().emoe_kv_append(p, layer, k, v, ks, vs, io, slots, n, None)
    return B.lib().emoe_kv_gather(p, layer, slots, n, k, v, ks, vs, io, None)


REFUSED = [
    (dict(arena=None), 1), (dict(layer=-1), 1), (dict(layer=2), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(slots=None), 1),
    (dict(n=-1), 1), (dict(io=3), 1), (dict(io=-1), 1), (dict(type=2), 1), (dict(type=4), 1), (dict(layout=1), 1), (dict(reserved=1), 1),
    (dict(scales=1 << 20), 1), (dict(type=3), 1),                       # scales with 16 bits, e4m3 without
    (dict(n_layers=0), 2), (dict(num_blocks=0), 2), (dict(block_tokens=-1), 2), (dict(n_heads=0), 2), (dict(head_dim=0), 2),
    (dict(num_blocks=1 << 30, block_tokens=2), 2), (dict(ks=31), 2), (dict(vs=16), 2),
    (dict(num_blocks=(1 << 31) - 1, block_tokens=1, n_heads=1 << 20, head_dim=1 << 20), 2),
    (dict(arena=(1 << 24) + 8), 5), (dict(k=(1 << 20) + 8), 5), (dict(v=(1 << 20) + 2), 5), (dict(slots=(1 << 20) + 4), 5),
    (dict(ks=33), 5), (dict(vs=36), 5), (dict(status=2), 5),
    (dict(io=1), 9), (dict(head_dim=12), 9), (dict(head_dim=264, ks=1000, vs=1000), 9),
    (dict(n=(1 << 31) - 1), 11),
]


@pytest.mark.parametrize("fn", ["emoe_kv_append", "emoe_kv_gather"])
@pytest.mark.parametrize("change,code", REFUSED)
def test_refusals(fn, change, code):
    assert _call(fn, **change) == code


def test_null_cache_and_empty_calls():
    assert _call(cache=ctypes.POINTER(B._KvCache)()) == 1
    for fn in ("emoe_kv_append", "emoe_kv_gather"):
        assert _call(fn, n=0, k=None, v=None, slots=None) == 0      # no token: nothing is looked at, no device needed


@pytest.mark.skipif(torch.cuda.is_available(), reason="looks at the answer without a device")
def test_without_a_device_the_call_is_refused():
    assert _call() == 8


def test_python_checks():
    make = lambda **kw: E.KvCache(torch.zeros(10000, dtype=torch.uint8), **{**DIMS, **kw})   # noqa: E731
    c = make()
    k, slots = torch.zeros(3, 2, 16, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="at least"):
        E.KvCache(torch.zeros(100, dtype=torch.uint8), **DIMS)
    for kw in (dict(kv_type="e4m3"), dict(scales=1 << 20), dict(kv_type="int8")):
        with pytest.raises(ValueError):
            make(**kw)
    for args in ((k[:2], k, slots), (k, k[:, :1], slots), (k.float(), k, slots), (k, k, slots.int()), (k, k, slots[None]),
                 (k.double(), k.double(), slots), (k.transpose(1, 2).contiguous().transpose(1, 2), k, slots)):
        with pytest.raises(ValueError):
            c.append(0, *args)
    with pytest.raises(E.EmoeError):
        E.KvCache(1 << 20, **{**DIMS, "n_heads": 0})


def test_reference_quantiser():
    """Hand-written points of the definition the GPU tests compare with."""
    x = np.zeros((7, 8))
    x[0, :3] = 448, -1, 0.3            # 448 is the largest code: k = 0
    x[1, 0] = 449                      # just above: k = 1, 224.5 lies between 224 and 240
    x[2] = 0
    x[3, 0] = np.inf
    x[4, 1] = np.nan
    x[5, :2] = 448, 18                 # 18 is a code, so is 17's even neighbour 16
    x[5, 2:4] = 17, 19                 # ties: to the even mantissa, 16 and 20
    x[6, 0] = 2.0 ** -140
    codes, b = R.quantise(x)
    assert list(b) == [127, 128, 127, 255, 255, 127, 1]
    assert codes[0, 0] == 448 and codes[0, 1] == -1 and codes[0, 2] == 0.3125 and codes[1, 0] == 224
    assert list(codes[5, :4]) == [448, 18, 16, 20] and not codes[3].any() and not codes[4].any()
    assert codes[6, 0] == 0
