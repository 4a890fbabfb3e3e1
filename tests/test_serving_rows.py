"""Refusals and workspaces of emoe_kv_extend, _keep, _attend_tree and _attend_window, on the CPU; their plain definitions against
each other and against plain softmax."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
import rows_ref as RR
import serving_ref as R
from paper_2510_02613_b200 import binding as B


def _cache(**changes):
    c = B._KvCache(1 << 24, None, None, 2, 30, 4, 2, 64, 0, 0, 0)
    for name, value in changes.items():
        setattr(c, name, value)
    return c


def _set(p, changes):
    for name, value in changes.items():
        assert hasattr(p, name)
        setattr(p, name, value)
    return p


def _rows(tree, layer=0, cache=None, **changes):
    p = _set(B._AttendRows(1 << 20, 1 << 21, None, 512, 512, 1 << 22, 1 << 23, 1 << 25, 1 << 26 if tree else None, 1 << 28, 1 << 40,
                           3, 40, 33, 8, 5, 2 if tree else 0, 0 if tree else 100, 0 if tree else 4, 0, 0.125, 0, 0), changes)
    call = B.lib().emoe_kv_attend_tree if tree else B.lib().emoe_kv_attend_window
    return call(ctypes.byref(_cache(**(cache or {}))), layer, ctypes.byref(p), None)


BOTH = [
    (dict(cache=dict(arena=None)), 1), (dict(layer=2), 1), (dict(layer=-1), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(block_table=None), 1),
    (dict(own_lens=None), 1), (dict(q_start=None), 1), (dict(reserved=1), 1), (dict(wait_limit_us=-2), 1), (dict(io_type=2), 1), (dict(io_type=3), 1),
    (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(n_seqs=-1), 2), (dict(n_tokens=-1), 2), (dict(max_q=0), 2),
    (dict(n_q_heads=0), 2), (dict(n_q_heads=7), 2), (dict(max_blocks=-1), 2), (dict(q_stride=511), 2), (dict(out_stride=64), 2),
    (dict(q=(1 << 20) + 8), 5), (dict(out=(1 << 20) + 2), 5), (dict(lse=2), 5), (dict(block_table=3), 5), (dict(own_lens=1), 5),
    (dict(q_start=(1 << 25) + 2), 5), (dict(workspace=(1 << 28) + 16), 5), (dict(q_stride=516), 5), (dict(out_stride=517), 5),
    (dict(io_type=1), 9), (dict(cache=dict(head_dim=48)), 9), (dict(cache=dict(head_dim=512)), 9),
    (dict(n_seqs=1 << 21), 11), (dict(n_tokens=1 << 25), 11), (dict(max_blocks=1 << 28), 11), (dict(n_tokens=1 << 24, n_q_heads=32), 11),
]


@pytest.mark.parametrize("change,code", BOTH + [(dict(mask=None), 1), (dict(mask=3), 5), (dict(mask_words=1), 2), (dict(window=1), 2), (dict(sinks=1), 2)])
def test_tree_refusals(change, code):
    assert _rows(True, **change) == code


@pytest.mark.parametrize("change,code", BOTH + [(dict(mask=1 << 20), 1), (dict(mask_words=1), 1), (dict(window=0), 2), (dict(sinks=-1), 2)])
def test_window_refusals(change, code):
    assert _rows(False, **change) == code


def test_too_small_a_workspace():
    need = ctypes.c_uint64()
    c = _cache(num_blocks=5000)
    assert B.lib().emoe_kv_attend_tree_workspace(ctypes.byref(c), 1, 8, 8, 8, 1000, ctypes.byref(need)) == 0 and need.value > 0
    one = dict(n_seqs=1, n_tokens=8, max_q=8, max_blocks=1000, mask_words=1, cache=dict(num_blocks=5000))
    assert _rows(True, workspace=None, **one) == 1
    assert _rows(True, workspace_bytes=8, **one) == 1


@pytest.mark.skipif(torch.cuda.is_available(), reason="looks at the answer without a device")
def test_without_a_device_the_calls_are_refused():
    assert _rows(True) == 8 and _rows(False) == 8 and _extend() == 8 and _keep() == 8


def test_empty_batches_do_nothing():
    for tree in (True, False):
        assert _rows(tree, n_seqs=0, q=None, out=None) == 0
        assert _rows(tree, n_tokens=0, q=None, out=None) == 0
    assert _keep(n_seqs=0, lens=None) == 0


def _extend(cache=None, **changes):
    p = _set(B._Extend(*((1 << 20) + 4096 * i for i in range(9)), 3, 5, 100, 64, 0, 0), changes)
    return B.lib().emoe_kv_extend(ctypes.byref(_cache(**(cache or {}))), ctypes.byref(p), None)


@pytest.mark.parametrize("change,code", [
    (dict(reserved=1), 1), (dict(reserved2=1), 1), (dict(lens=None), 1), (dict(add=None), 1), (dict(block_table=None), 1), (dict(free_blocks=None), 1),
    (dict(n_free=None), 1), (dict(q_start=None), 1), (dict(slots=None), 1), (dict(lens_out=None), 1), (dict(n_free_out=None), 1),
    (dict(n_seqs=-1), 2), (dict(max_blocks=-1), 2), (dict(free_capacity=-1), 2), (dict(n_slots=-1), 2), (dict(n_seqs=8193), 11),
    (dict(max_blocks=1 << 28), 11), (dict(n_seqs=8192, max_blocks=1 << 18), 11), (dict(slots=(1 << 20) + 4), 5), (dict(lens=2), 5),
    (dict(add=1), 5), (dict(q_start=3), 5), (dict(n_free_out=6), 5), (dict(cache=dict(num_blocks=0)), 2), (dict(cache=dict(type=2)), 1),
])
def test_extend_refusals(change, code):
    assert _extend(**change) == code


def _keep(cache=None, **changes):
    p = _set(B._Keep(*((1 << 20) + 4096 * i for i in range(6)), 3, 5, 4, 0), changes)
    return B.lib().emoe_kv_keep(ctypes.byref(_cache(**(cache or {}))), ctypes.byref(p), None)


@pytest.mark.parametrize("change,code", [
    (dict(reserved=1), 1), (dict(lens=None), 1), (dict(block_table=None), 1), (dict(q_start=None), 1), (dict(accepted=None), 1),
    (dict(n_accepted=None), 1), (dict(change=None), 1), (dict(cache=dict(arena=None)), 1), (dict(cache=dict(type=3)), 1), (dict(n_seqs=-1), 2),
    (dict(max_blocks=-1), 2), (dict(max_accepted=-1), 2), (dict(cache=dict(head_dim=20)), 9), (dict(n_seqs=1 << 16), 11),
    (dict(max_accepted=1025), 11), (dict(max_blocks=1 << 28), 11), (dict(lens=2), 5), (dict(change=2), 5), (dict(accepted=1), 5),
])
def test_keep_refusals(change, code):
    assert _keep(**change) == code


def test_null_structs():
    c, n = _cache(), ctypes.c_uint64()
    L = B.lib()
    for call in (L.emoe_kv_attend_tree, L.emoe_kv_attend_window):
        assert call(ctypes.byref(c), 0, None, None) == 1 and call(None, 0, None, None) == 1
    for call in (L.emoe_kv_extend, L.emoe_kv_keep):
        assert call(ctypes.byref(c), None, None) == 1 and call(None, None, None) == 1
    assert L.emoe_kv_attend_tree_workspace(ctypes.byref(c), 1, 1, 1, 2, 1, None) == 1
    assert L.emoe_kv_attend_window_workspace(ctypes.byref(c), 1, 1, 1, 2, 1, 0, 0, ctypes.byref(n)) == 2
    assert L.emoe_kv_attend_window_workspace(None, 1, 1, 1, 2, 1, 1, 0, ctypes.byref(n)) == 1


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("hd", [32, 64, 128, 256])
def test_workspaces_grow(kv, hd):
    """Enough for a call is enough for calls with less of any size: what smaller calls refuse must not be what the bound gives."""
    rng = np.random.default_rng(hd)
    c = _cache(num_blocks=100000, block_tokens=16, n_heads=4, head_dim=hd, type=3 if kv == "e4m3" else 0, scales=1 << 30 if kv == "e4m3" else None)
    n = ctypes.c_uint64()

    def need(n_seqs, n_tokens, max_q, hq, blocks, window, sinks):
        assert B.lib().emoe_kv_attend_window_workspace(ctypes.byref(c), n_seqs, n_tokens, max_q, hq, blocks, window, sinks, ctypes.byref(n)) == 0
        return n.value

    def accepted(size, have):
        n_seqs, n_tokens, max_q, hq, blocks, window, sinks = size
        p = B._AttendRows(1 << 20, 1 << 21, None, 1 << 20, 1 << 20, 1 << 22, 1 << 23, 1 << 25, None, 1 << 28 if have else None, have,
                          n_seqs, n_tokens, max_q, hq, blocks, 0, window, sinks, 0, 0.125, 0, 0)
        return B.lib().emoe_kv_attend_window(ctypes.byref(c), 0, ctypes.byref(p), None) != 1

    for _ in range(200):
        big = [int(2 ** rng.uniform(0, 7)), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 13)), 4 * int(rng.integers(1, 9)),
               int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 15)), int(rng.integers(0, 100))]
        have = need(*big)
        assert accepted(big, have)
        for _ in range(10):
            small = [int(rng.integers(1, max(1, x) + 1)) for x in big]
            small[3] = 4 * int(rng.integers(1, big[3] // 4 + 1))
            small[6] = int(rng.integers(0, big[6] + 1))
            assert need(*small) <= have and accepted(small, have), (big, small)


def test_workspaces_of_trees_grow():
    rng = np.random.default_rng(5)
    c, n = _cache(num_blocks=100000, block_tokens=16, n_heads=4, head_dim=128), ctypes.c_uint64()

    def need(*size):
        assert B.lib().emoe_kv_attend_tree_workspace(ctypes.byref(c), *size, ctypes.byref(n)) == 0
        return n.value
    for _ in range(200):
        big = [int(2 ** rng.uniform(0, 7)), int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 8)), 4 * int(rng.integers(1, 9)), int(2 ** rng.uniform(0, 12))]
        have = need(*big)
        for _ in range(10):
            small = [int(rng.integers(1, x + 1)) for x in big]
            small[3] = 4 * int(rng.integers(1, big[3] // 4 + 1))
            p = B._AttendRows(1 << 20, 1 << 21, None, 1 << 20, 1 << 20, 1 << 22, 1 << 23, 1 << 25, 1 << 26, 1 << 28 if have else None, have, *small, 8, 0, 0, 0, 0.125, 0, 0)
            assert need(*small) <= have and B.lib().emoe_kv_attend_tree(ctypes.byref(c), 0, ctypes.byref(p), None) != 1, (big, small)


def test_python_checks():
    arena = torch.zeros(2 * 8 * 4 * 2 * 64 * 2, dtype=torch.uint8)
    c = E.KvCache(arena, n_layers=1, num_blocks=8, block_tokens=4, n_heads=2, head_dim=64)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)    # noqa: E731
    q = torch.zeros(6, 4, 64, dtype=torch.bfloat16)
    good = dict(q=q, out=q.clone(), block_table=i32(3, 2), own_lens=i32(3), q_start=i32(4), max_q=4)
    bads = (dict(q=q[..., :32]), dict(out=q.float()), dict(out=q[:2]), dict(block_table=i32(2, 2)), dict(block_table=i32(3, 2).long()), dict(own_lens=i32(2)),
            dict(q_start=i32(3)), dict(q_start=i32(4).long()), dict(own_lens=None), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)),
            dict(lse=torch.zeros(3, 4)), dict(q=q.double(), out=q.double()), dict(block_table=i32(2, 3).T))
    for bad in bads + (dict(mask=i32(5, 1)), dict(mask=i32(6, 1).float()), dict(mask=i32(6, 2)[:, :1]), dict(mask=None)):
        with pytest.raises(ValueError):
            c.attend_tree(0, **{**good, "mask": i32(6, 1), **bad})
    for bad in bads:
        with pytest.raises(ValueError):
            c.attend_window(0, **{**good, "window": 3, **bad})
    good = dict(lens=i32(3), add=i32(3), block_table=i32(3, 2), free_blocks=i32(9), n_free=i32(1), q_start=i32(4), slots=i32(7).long(),
                lens_out=i32(3), n_free_out=i32(1))
    for bad in (dict(lens=i32(3).long()), dict(add=i32(2)), dict(block_table=i32(2, 2)), dict(n_free=i32(2)), dict(q_start=i32(3)), dict(slots=i32(7)),
                dict(lens_out=i32(2)), dict(n_free_out=i32(1).long()), dict(free_blocks=i32(9, 1)), dict(lens=i32(6)[::2]), dict(slots=None)):
        with pytest.raises(ValueError):
            c.extend(**{**good, **bad})
    good = dict(block_table=i32(3, 2), lens=i32(3), q_start=i32(4), accepted=i32(3, 5), n_accepted=i32(3), change=i32(3))
    for bad in (dict(block_table=i32(3)), dict(lens=i32(3).long()), dict(q_start=i32(3)), dict(accepted=i32(2, 5)), dict(n_accepted=i32(4)), dict(change=None),
                dict(accepted=i32(5, 3).T)):
        with pytest.raises(ValueError):
            c.keep(**{**good, **bad})


def test_masks_of_the_definitions():
    assert RR.window_sees(6, 2, 2, 1).tolist() == [[True, False, False, True, True, False], [True, False, False, False, True, True]]
    assert RR.window_sees(2, 3, 1, 0).tolist() == [[False, False], [True, False], [False, True]]
    bits = np.array([[1, 0, 0], [1, 1, 0], [1, 0, 1]], bool)
    assert RR.tree_sees(5, 3, bits).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 0, 1]]
    assert RR.tree_sees(2, 3, bits).tolist() == [[0, 0], [1, 0], [0, 1]]
    assert RR.packed_bits(np.eye(40, dtype=bool), 2)[[0, 31, 35]].tolist() == [[1, 0], [-2 ** 31, 0], [0, 8]]


def test_attention_of_the_definitions_against_softmax():
    rng = np.random.default_rng(0)
    ref = R.Cache(1, 5, 3, 2, 8, "f16")
    ref.values = rng.standard_normal(ref.values.shape)
    table = np.array([[4, 1], [0, -1]], np.int32)
    q = torch.from_numpy(rng.standard_normal((3, 4, 8)))
    sees = [RR.window_sees(5, 2, 2, 1), RR.window_sees(1, 1, 2, 1)]
    o, lse, _, _, _ = RR.attend(ref, 0, q, table, [5, 1], [0, 2, 3], sees, 0.3)
    flat = ref.values[0].reshape(2, 15, 2, 8)
    for row, seen in ((0, [12, 14, 3]), (1, [12, 3, 4]), (2, [0])):
        for h in range(4):
            k, v = torch.from_numpy(flat[0, seen, h // 2]), torch.from_numpy(flat[1, seen, h // 2])
            score = 0.3 * (k @ q[row, h])
            assert np.allclose(o[row, h], torch.softmax(score, 0) @ v, atol=1e-12)
            assert np.isclose(lse[row, h], torch.logsumexp(score, 0))


def test_extend_of_the_definition():
    # blocks of 4; sequence 0 grows into a block, 1 gives one back, 2 stays, 3 wants more than there is
    out, table, free, left, start, slots, status = RR.extend([4, 9, 3, 0], [2, -3, 0, 9], [[7, -1, -1], [1, 2, 3], [5, -1, -1], [-1, -1, -1]],
                                                             [8, 9, -1, -1], 2, 20, 4, 10)
    assert out == [6, 6, 3, 0] and start == [0, 2, 2, 2, 11] and left == 2 and status == 11
    assert table[0] == [7, 3, -1] and table[3] == [-1, -1, -1] and free == [8, 9, 3, -1]
    assert slots[:3] == [12, 13, -1] and set(slots[2:]) == {-1}
