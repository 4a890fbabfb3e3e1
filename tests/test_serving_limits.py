"""Refusals, sizes and checks of the serving operators on the CPU, beside those of test_serving_*.py."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2510_02613_b200 as E
from paper_2510_02613_b200 import binding as B
from test_serving_attend import _call as attend
from test_serving_kv import _call as copy


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


def _sizes(rng, heads):
    log = lambda lo, hi: int(2.0 ** rng.uniform(np.log2(lo), np.log2(hi)))    # noqa: E731
    return [log(1, 400), int(rng.integers(1, 5)), heads * log(1, 17), log(1, 300) if rng.random() < 0.8 else 0,
            log(1, 200000) if rng.random() < 0.7 else 0]


@pytest.mark.parametrize("head_dim,kv", [(128, "bf16"), (64, "e4m3"), (256, "bf16"), (32, "e4m3")])
def test_an_attention_workspace_is_enough_for_smaller_calls(head_dim, kv):
    rng = np.random.default_rng(head_dim)
    for _ in range(1200):
        heads, block = int(2 ** rng.integers(0, 6)), int(rng.choice([1, 7, 16, 64]))
        scales = (1 << 24) if kv == "e4m3" else None
        c = E.KvCache(1 << 24, n_layers=1, num_blocks=1 << 20, block_tokens=block, n_heads=heads, head_dim=head_dim, kv_type=kv, scales=scales)
        raw = B._KvCache(1 << 24, scales, None, 1, 1 << 20, block, heads, head_dim, c.kv_type, 0, 0)
        size = _sizes(rng, heads)
        bytes_ = c.attend_workspace_bytes(*size)
        assert bytes_ <= 16 * 520 * (9 << 20)     # and not out of all proportion
        for _ in range(40):
            less = [int(x * 2.0 ** -rng.uniform(0, 8 * (rng.random() < 0.5))) for x in size]
            less = [max(1, less[0]), max(1, less[1]), max(heads, less[2] // heads * heads)] + less[3:]
            assert c.attend_workspace_bytes(*less) <= bytes_
            n, t, hq, blocks, prefix = less
            p = B._Attend(1 << 20, 1 << 21, None, hq * head_dim, hq * head_dim, 1 << 22, 1 << 23, 1 << 25, 1 << 28, bytes_, n, t, hq, blocks,
                          prefix, 0, 0.125, 0)
            # refused for the arena, which is no memory of a device, and not for the workspace
            assert B.lib().emoe_kv_attend(ctypes.byref(raw), 0, ctypes.byref(p), None) == 8, (size, less)


def test_attention_workspaces_of_usual_calls():
    c = E.KvCache(1 << 20, n_layers=1, num_blocks=50000, block_tokens=16, n_heads=4, head_dim=128)
    mib = [c.attend_workspace_bytes(*x) / 2 ** 20 for x in ((128, 1, 32, 172, 65536), (64, 1, 32, 172, 0), (1, 1, 32, 512, 0), (1, 1, 32, 4, 0))]
    assert mib[0] < 80 and mib[1] < 25 and mib[2] < 2 and mib[3] == 0


def _handles(arena):
    """(cache, its attend arguments, experts, their decode arguments), tensors on the CPU."""
    size = 2 * 8 * 4 * 2 * 64 * 2
    cache = E.KvCache(torch.zeros(size, dtype=torch.uint8) if arena is None else arena, n_layers=1, num_blocks=8, block_tokens=4, n_heads=2, head_dim=64)
    q, table = torch.zeros(3, 1, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, dtype=torch.int32)
    attend_args = dict(q=q, out=q.clone(), block_table=table, own_lens=torch.zeros(3, dtype=torch.int32))
    experts = E.ExpertArena(torch.zeros(3 * 6 * 64 * 32 * 2, dtype=torch.uint8) if arena is None else arena, n_layers=1, n_slots=6, d_model=64, d_ff=32)
    x = torch.zeros(3, 64, dtype=torch.bfloat16)
    decode_args = dict(x=x, logits=torch.zeros(3, 8), top_k=2, slot_of_expert=torch.zeros(8, dtype=torch.int32), out=x.clone())
    return cache, attend_args, experts, decode_args


def test_workspaces_are_checked():
    """A workspace has to lie where the arena does, in one piece."""
    cache, a, experts, d = _handles(None)
    for work in (torch.empty(1 << 20, dtype=torch.uint8, device="meta"), torch.empty(1 << 20, dtype=torch.uint8)[::2],
                 torch.empty(1, dtype=torch.uint8).expand(1 << 20)):
        with pytest.raises(ValueError, match="workspace"):
            cache.attend(0, **a, workspace=work)
        with pytest.raises(ValueError, match="workspace"):
            experts.decode(0, **d, workspace=work)


def test_tensors_beside_an_arena_given_as_an_address():
    """Nothing says where it lies; a CPU tensor is refused all the same, before its address reaches a kernel."""
    cache, a, experts, d = _handles(1 << 24)
    k, slots = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="cpu"):
        cache.attend(0, **a)
    with pytest.raises(ValueError, match="cpu"):
        cache.append(0, k, k, slots)
    with pytest.raises(ValueError, match="cpu"):
        cache.gather(0, slots, k, k.clone())
    with pytest.raises(ValueError, match="cpu"):
        experts.decode(0, **d)


def test_a_status_word_tells_where_an_arena_lies():
    status = torch.zeros(1, dtype=torch.int32, device="meta")
    cache = E.KvCache(1 << 24, n_layers=1, num_blocks=8, block_tokens=4, n_heads=2, head_dim=64, status=status)
    assert cache.device == status.device
    with pytest.raises(ValueError, match="cpu"):
        cache.append(0, torch.zeros(1, 2, 64), torch.zeros(1, 2, 64), torch.zeros(1, dtype=torch.int64, device="meta"))


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 3e38, -3e38])
def test_an_attention_scale_is_finite(scale):
    """The two kernels would answer such calls differently.  (3e38 is not finite any more as a factor of exponents of 2.)"""
    assert attend(scale=scale) == 1


@pytest.mark.parametrize("fn", ["emoe_kv_append", "emoe_kv_gather"])
def test_places_inside_a_token_fit_32_bits(fn):
    big = dict(n_heads=1 << 23, head_dim=128, num_blocks=1, ks=1 << 30, vs=1 << 30)
    for n in (1, 2):
        assert copy(fn, io=2, n=n, **big) == 11            # 4 GB a token
        assert copy(fn, io=0, n=n, **big) == 8             # 2 GB: refused for the arena only


def test_missing_tensors_are_named():
    cache, a, _, _ = _handles(None)
    for bad, what in ((dict(own_lens=None), "own_lens"), (dict(block_table=None), "block_table"), (dict(prefix_len=5), "prefix_table")):
        with pytest.raises(ValueError, match=what + " is missing"):
            cache.attend(0, **{**a, **bad})
