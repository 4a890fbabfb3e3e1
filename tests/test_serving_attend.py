"""Refusals and workspace of emoe_kv_attend, on the CPU; the 64-bit reference against plain softmax."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import serving_ref as R
from paper_2510_02613_b200 import binding as B


def _call(layer=0, cache=None, **changes):
    c = B._KvCache(1 << 24, None, None, 2, 30, 4, 2, 64, 0, 0, 0)
    p = B._Attend(1 << 20, 1 << 21, None, 512, 512, 1 << 22, 1 << 23, 1 << 25, 1 << 28, 1 << 40, 3, 1, 8, 5, 9, 0, 0.125, 0)
    for name, value in changes.items():
        setattr(c if hasattr(c, name) and name not in ("reserved",) else p, name, value)
    for name, value in (cache or {}).items():
        setattr(c, name, value)
    return B.lib().emoe_kv_attend(ctypes.byref(c), layer, ctypes.byref(p), None)


@pytest.mark.parametrize("change,code", [
    (dict(arena=None), 1), (dict(layer=2), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(block_table=None), 1), (dict(own_lens=None), 1),
    (dict(prefix_table=None), 1), (dict(reserved=1), 1), (dict(io_type=2), 1), (dict(io_type=3), 1), (dict(workspace=None), 1),
    (dict(workspace_bytes=8), 1), (dict(n_seqs=-1), 2), (dict(q_len=0), 2), (dict(n_q_heads=0), 2), (dict(n_q_heads=7), 2),
    (dict(max_blocks=-1), 2), (dict(prefix_len=-1), 2), (dict(q_stride=511), 2), (dict(out_stride=64), 2),
    (dict(q=(1 << 20) + 8), 5), (dict(out=(1 << 20) + 2), 5), (dict(lse=2), 5), (dict(block_table=3), 5), (dict(own_lens=1), 5),
    (dict(prefix_table=2), 5), (dict(workspace=(1 << 28) + 16), 5), (dict(q_stride=516), 5), (dict(out_stride=517), 5),
    (dict(io_type=1), 9), (dict(head_dim=48), 9), (dict(head_dim=512), 9),
    (dict(n_seqs=1 << 25), 11), (dict(q_len=1 << 24), 11), (dict(max_blocks=1 << 28), 11), (dict(prefix_len=1 << 30), 11),
])
def test_refusals(change, code):
    assert _call(**change) == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="looks at the answer without a device")
def test_without_a_device_the_call_is_refused():
    assert _call() == 8


def test_an_empty_batch_does_nothing():
    assert _call(n_seqs=0, q=None, out=None) == 0


def test_null_structs():
    c = B._KvCache(1 << 24, None, None, 2, 30, 4, 2, 64, 0, 0, 0)
    assert B.lib().emoe_kv_attend(ctypes.byref(c), 0, None, None) == 1
    assert B.lib().emoe_kv_attend(None, 0, None, None) == 1
    assert B.lib().emoe_kv_attend_workspace(ctypes.byref(c), 1, 1, 2, 1, 0, None) == 1


def test_workspace_sizes():
    c = E.KvCache(1 << 20, n_layers=1, num_blocks=5000, block_tokens=16, n_heads=4, head_dim=128)
    assert c.attend_workspace_bytes(0, 1, 32, 10, 0) == 0
    assert c.attend_workspace_bytes(1, 1, 32, 1, 0) == 0              # one part: nothing to join
    for n, t, blocks, prefix in ((1, 1, 200, 0), (48, 1, 47, 2000), (128, 4, 47, 65536), (3, 2, 0, 1000)):
        need = c.attend_workspace_bytes(n, t, 32, blocks, prefix)
        assert 0 <= need <= n * t * 32 * 128 * (128 * 4 + 8) + 512 and need % 256 == 0
    with pytest.raises(E.EmoeError):
        c.attend_workspace_bytes(1, 1, 30, 1, 0)


def test_python_checks():
    arena = torch.zeros(2 * 8 * 4 * 2 * 64 * 2, dtype=torch.uint8)
    c = E.KvCache(arena, n_layers=1, num_blocks=8, block_tokens=4, n_heads=2, head_dim=64)
    q = torch.zeros(3, 1, 4, 64, dtype=torch.bfloat16)
    table, lens, pt = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    good = dict(q=q, out=q.clone(), block_table=table, own_lens=lens, prefix_table=pt, prefix_len=8)
    for bad in (dict(q=q[..., :32]), dict(out=q.float()), dict(out=q[:2]), dict(block_table=table[:2]), dict(block_table=table.long()),
                dict(own_lens=lens[:2]), dict(own_lens=lens.long()), dict(prefix_len=9), dict(prefix_table=pt.long()),
                dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), dict(lse=torch.zeros(3, 4)), dict(q=q.double())):
        with pytest.raises(ValueError):
            c.attend(0, **{**good, **bad})


def test_reference_against_softmax():
    rng = np.random.default_rng(0)
    ref = R.Cache(1, 5, 3, 2, 8, "f16")
    ref.values = rng.standard_normal(ref.values.shape)
    table, pt = np.array([[4, 1], [0, -1]], np.int32), np.array([2, 3], np.int32)
    q = rng.standard_normal((2, 2, 4, 8))
    o, lse, _, _ = R.attend(ref, 0, q, table, [5, 1], pt, 4, 0.3)
    flat = ref.values[0].reshape(2, 15, 2, 8)
    for s, own in ((0, [12, 13, 14, 3, 4]), (1, [0])):
        for t in range(2):
            seen = [6, 7, 8, 9] + own[:len(own) - 1 + t]
            for h in range(4):
                k, v = torch.from_numpy(flat[0, seen, h // 2]), torch.from_numpy(flat[1, seen, h // 2])
                score = 0.3 * (k @ torch.from_numpy(q[s, t, h]))
                assert np.allclose(o[s, t, h], torch.softmax(score, 0) @ v, atol=1e-12)
                assert np.isclose(lse[s, t, h], torch.logsumexp(score, 0))
