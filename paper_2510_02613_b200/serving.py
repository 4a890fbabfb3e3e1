"""Operators that serve from one rank's arenas between two scale steps: the handles below describe
an arena as the library lays it out and marshal torch tensors to the C entry points, which only
enqueue on the stream they are given (None: the legacy default stream, as for the reshard calls).

Tensors are checked for type, shape and device here; ids and lengths that lie in device memory are
bounds-checked by the kernels (see emoe_kv_cache_t.status)."""
from __future__ import annotations

import ctypes
from typing import Optional

from . import binding as _b
from .binding import _check, _stream_handle

BF16, F16, F32, E4M3 = range(4)
_TYPE_NAMES = {"bf16": BF16, "f16": F16, "e4m3": E4M3}
_TORCH_TYPES = {"torch.bfloat16": BF16, "torch.float16": F16, "torch.float32": F32}
_TYPE_BYTES = {BF16: 2, F16: 2, F32: 4, E4M3: 1}


def _type_of(name: str) -> int:
    try:
        return _TYPE_NAMES[name]
    except KeyError:
        raise ValueError("element type %r: one of %s" % (name, ", ".join(_TYPE_NAMES))) from None


_types: dict = {}   # torch dtype -> type, filled as they come (their names are slow to make)


def _value_type(t, what: str) -> int:
    code = _types.get(t.dtype)
    if code is None:
        code = _types[t.dtype] = _TORCH_TYPES.get(str(t.dtype), -1)
    if code < 0:
        raise ValueError("%s: bfloat16, float16 or float32, not %s" % (what, t.dtype))
    return code


_names: dict = {}   # torch dtype -> its name


def _placed(t, what: str, device) -> None:
    """ValueError unless t lies where the arena does (device None: the arena was given as an address, which the
    call itself looks for on the current device)."""
    if device is None:
        if not t.is_cuda:
            raise ValueError("%s is on %s, the arena on a CUDA device" % (what, t.device))
        import torch
        if t.get_device() != torch.cuda.current_device():
            raise ValueError("%s is on %s, which is not the current device" % (what, t.device))
    elif t.device != device:
        raise ValueError("%s is on %s, the arena on %s" % (what, t.device, device))


def _shaped(t, what: str, shape, dtype: Optional[str], device):
    """t itself; ValueError unless it has this shape (None: any size), type and place."""
    if t is None:
        raise ValueError("%s is missing" % what)
    if len(t.shape) != len(shape) or any(w is not None and w != n for n, w in zip(t.shape, shape)):
        raise ValueError("%s: shape %s, wanted %s" % (what, tuple(t.shape), tuple("any" if w is None else w for w in shape)))
    if dtype is not None:
        name = _names.get(t.dtype)
        if name is None:
            name = _names[t.dtype] = str(t.dtype)[6:]
        if name != dtype:
            raise ValueError("%s: %s, wanted %s" % (what, name, dtype))
    _placed(t, what, device)
    return t


def _dense(t, what: str, inner: int):
    """t itself; ValueError unless its last `inner` dimensions are densely packed."""
    if t.is_contiguous():
        return t
    step = 1
    for n, s in list(zip(t.shape, t.stride()))[:-inner - 1:-1]:
        if n != 1 and s != step:
            raise ValueError("%s: its last %d dimensions have to be contiguous" % (what, inner))
        step *= n
    return t


def _dense_pointer(t, what: str, shape, dtype: str, device):
    """Address of a tensor of this shape (None: any size) and type, densely packed, beside the arena; ValueError otherwise.
    (The first test is what a good call pays.)"""
    if t is None or t.shape != shape or _names.get(t.dtype) != dtype or t.device != device or not t.is_contiguous():
        _dense(_shaped(t, what, shape, dtype, device), what, len(shape))
    return t.data_ptr()


def _sizes(t, what: str, n: int):
    """The n sizes of t; ValueError if it has not as many."""
    if t is None or t.dim() != n:
        raise ValueError("%s: %s, wanted a tensor of %d dimensions" % (what, "missing" if t is None else tuple(t.shape), n))
    return t.shape


def _workspace(t, device):
    """(address, bytes) of a workspace or None."""
    if t is None:
        return None, 0
    _placed(t, "workspace", device)
    if not t.is_contiguous():
        raise ValueError("workspace: not contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def _arena_pointer(arena, need: int, what: str):
    """(address, device or None): a tensor has to be large enough and contiguous; an address is taken as it is."""
    if isinstance(arena, int):
        return arena, None
    if not arena.is_contiguous():
        raise ValueError("%s: not contiguous" % what)
    if arena.numel() * arena.element_size() < need:
        raise ValueError("%s: %d bytes, at least %d are needed" % (what, arena.numel() * arena.element_size(), need))
    return arena.data_ptr(), arena.device


class KvCache:
    """One rank's paged KV cache: emoe_kv_append, emoe_kv_gather, emoe_kv_attend, emoe_kv_extend, emoe_kv_attend_tree,
    emoe_kv_attend_window, emoe_kv_keep.

    arena: tensor or device address, [n_layers][2][num_blocks][block_tokens][n_heads][head_dim] as
    emoe_reshard_kv lays it out (head_major: [n_heads][block_tokens] inside a block).  kv_type: "bf16",
    "f16" or "e4m3"; the last has scale bytes [n_layers][2][num_blocks][block_tokens][n_heads] in
    `scales`, a KV arena of head_dim 1 and elem_bytes 1.  status: optional int32 tensor of one element,
    set to 4 (EMOE_ERR_BLOCK_TABLE) by calls that meet an id outside the pool, to 10 (EMOE_ERR_DEVICE_TIMEOUT)
    by an attend whose bounded waits run out, to 11 (EMOE_ERR_TOO_LARGE) by an extend that refuses a sequence and by an
    attend_tree or attend_window that meets more than max_q query tokens."""

    def __init__(self, arena, *, n_layers: int, num_blocks: int, block_tokens: int, n_heads: int, head_dim: int,
                 kv_type: str = "bf16", scales=None, head_major: bool = False, status=None):
        self._c = _b._KvCache(None, None, None, n_layers, num_blocks, block_tokens, n_heads, head_dim, _type_of(kv_type),
                              _b.LAYOUT_KV_HEAD_MAJOR if head_major else 0, 0)
        self.kv_type, self.n_heads, self.head_dim, self.block_tokens = self._c.type, n_heads, head_dim, block_tokens
        sizes = self.bytes()
        self._c.arena, self.device = _arena_pointer(arena, sizes[0], "arena")
        if (scales is None) == (self.kv_type == E4M3):
            raise ValueError("an e4m3 cache has scales, another has none")
        if scales is not None:
            self._c.scales, device = _arena_pointer(scales, sizes[1], "scales")
            if None not in (device, self.device) and device != self.device:
                raise ValueError("scales are on %s, the arena on %s" % (device, self.device))
            self.device = self.device or device
        if status is not None:
            self.device = self.device or status.device
            self._c.status = _shaped(status, "status", (1,), "int32", self.device).data_ptr()
        self._keep = (arena, scales, status)
        self._ref = ctypes.byref(self._c)
        self._row = n_heads * head_dim
        L = self._calls = _b.lib()
        self._append, self._gather, self._attend = L.emoe_kv_append, L.emoe_kv_gather, L.emoe_kv_attend

    @classmethod
    def for_rank(cls, shape, tp: int, num_blocks: int, arena, kv_type: str = "bf16", **kw) -> "KvCache":
        """The cache of one of `tp` ranks of a model `shape`, as a plan with that shape lays it out."""
        if _TYPE_BYTES[_type_of(kv_type)] != shape.elem_bytes:
            raise ValueError("%s elements have %d bytes, the shape's %d" % (kv_type, _TYPE_BYTES[_type_of(kv_type)], shape.elem_bytes))
        return cls(arena, n_layers=shape.n_layers, num_blocks=num_blocks, block_tokens=shape.kv_block_tokens,
                   n_heads=max(1, shape.n_kv_heads // tp), head_dim=shape.head_dim, kv_type=kv_type, **kw)

    def bytes(self):
        """(bytes of the arena, bytes of the scales)"""
        a, s = ctypes.c_uint64(), ctypes.c_uint64()
        _check(_b.lib().emoe_kv_cache_bytes(ctypes.byref(self._c), ctypes.byref(a), ctypes.byref(s)))
        return a.value, s.value

    def vector_index(self, layer: int, kv: int, slot: int, head: int) -> int:
        """Index of a head vector in the arena (kv: 0 keys, 1 values), -1 if out of range."""
        return _b.lib().emoe_kv_vector_index(self._ref, layer, kv, slot, head)

    def _rows(self, x, what, n):
        if x.shape != (n, self.n_heads, self.head_dim) or x.device != self.device:
            _shaped(x, what, (n, self.n_heads, self.head_dim), None, self.device)
        if x.is_contiguous():
            return x.data_ptr(), self._row
        return _dense(x, what, 2).data_ptr(), (x.stride(0) if n > 1 else self._row)

    def _copy_args(self, k, v, slots):
        if not slots.is_contiguous():
            raise ValueError("slots: not contiguous")
        n = _shaped(slots, "slots", (None,), "int64", self.device).shape[0]
        (kp, ks), (vp, vs) = self._rows(k, "k", n), self._rows(v, "v", n)
        if k.dtype != v.dtype:
            raise ValueError("k is %s, v %s" % (k.dtype, v.dtype))
        return n, kp, ks, vp, vs, _value_type(k, "k")

    def append(self, layer: int, k, v, slots, stream=None) -> None:
        """Writes tokens' keys and values, [n, n_heads, head_dim] with any stride between tokens, into
        their slots (int64: block * block_tokens + offset; negative: skipped), quantising where the
        cache is e4m3."""
        n, kp, ks, vp, vs, t = self._copy_args(k, v, slots)
        _check(self._append(self._ref, layer, kp, vp, ks, vs, t, slots.data_ptr(), n, _stream_handle(stream)))

    def gather(self, layer: int, slots, k, v, stream=None) -> None:
        """Reads slots back into k and v; rows of negative slots stay as they were."""
        n, kp, ks, vp, vs, t = self._copy_args(k, v, slots)
        _check(self._gather(self._ref, layer, slots.data_ptr(), n, kp, vp, ks, vs, t, _stream_handle(stream)))

    def attend_workspace_bytes(self, n_seqs: int, q_len: int, n_q_heads: int, max_blocks: int, prefix_len: int = 0) -> int:
        """Enough for calls of up to these sizes on this cache."""
        n = ctypes.c_uint64()
        _check(_b.lib().emoe_kv_attend_workspace(self._ref, n_seqs, q_len, n_q_heads, max_blocks, prefix_len, ctypes.byref(n)))
        return n.value

    def attend(self, layer: int, q, out, block_table, own_lens, prefix_table=None, prefix_len: int = 0,
               scale: Optional[float] = None, lse=None, workspace=None, stream=None, wait_limit_us: int = 0) -> None:
        """Decode attention: q, out [n_seqs, q_len, n_q_heads, head_dim] (any stride between tokens); own
        tokens on the blocks of block_table [n_seqs, max_blocks] (int32), own_lens [n_seqs] of them (int32,
        the query tokens included; both None: prefix only); prefix_len tokens on the blocks of
        prefix_table, shared by all sequences.  workspace: attend_workspace_bytes bytes of the caller's,
        not shared by calls that can overlap.  lse: optional float32 [n_seqs, q_len, n_q_heads].
        wait_limit_us: bound of the waits inside the kernels (0: 4 s)."""
        n, t, hq, _ = q.shape
        _shaped(q, "q", (n, t, hq, self.head_dim), None, self.device)
        if out.dtype != q.dtype:
            raise ValueError("out is %s, q %s" % (out.dtype, q.dtype))
        _shaped(out, "out", (n, t, hq, self.head_dim), None, self.device)
        strides = [hq * self.head_dim] * 2
        for i, (x, what) in enumerate(((q, "q"), (out, "out"))):
            if not x.is_contiguous():
                _dense(x, what, 2)
                strides[i] = x.stride(1) if t > 1 else x.stride(0) if n > 1 else hq * self.head_dim
                if t > 1 and n > 1 and x.stride(0) != t * strides[i]:
                    raise ValueError("%s: sequences have to follow one another at the stride of the tokens" % what)
        blocks, bt, ol, pt = 0, None, None, None
        if block_table is not None or own_lens is not None:
            _dense(_shaped(block_table, "block_table", (n, None), "int32", self.device), "block_table", 2)
            _dense(_shaped(own_lens, "own_lens", (n,), "int32", self.device), "own_lens", 1)
            blocks, bt, ol = block_table.shape[1], block_table.data_ptr(), own_lens.data_ptr()
        if prefix_len > 0:
            _dense(_shaped(prefix_table, "prefix_table", (None,), "int32", self.device), "prefix_table", 1)
            if prefix_table.shape[0] * self.block_tokens < prefix_len:
                raise ValueError("prefix_table: %d blocks hold fewer than %d tokens" % (prefix_table.shape[0], prefix_len))
            pt = prefix_table.data_ptr()
        p = _b._Attend(q.data_ptr(), out.data_ptr(),
                       None if lse is None else _dense(_shaped(lse, "lse", (n, t, hq), "float32", self.device), "lse", 3).data_ptr(),
                       strides[0], strides[1], bt, ol, pt, *_workspace(workspace, self.device), n, t, hq, blocks, prefix_len,
                       _value_type(q, "q"), self.head_dim ** -0.5 if scale is None else scale, 0, wait_limit_us, 0)
        _check(self._attend(self._ref, layer, ctypes.byref(p), _stream_handle(stream)))

    def extend(self, lens, add, block_table, free_blocks, n_free, q_start, slots, lens_out, n_free_out, stream=None) -> None:
        """Blocks for a batch's next tokens, from lengths in device memory: sequence s of lens[s] tokens changes by
        add[s] (int32 [n] both), gets blocks from the end of free_blocks (int32; the first n_free [1] of it are free) into
        its row of block_table (int32 [n, max_blocks]) or gives them back (entries of -1 apart: blocks that were given back by hand,
        as those behind a window may be, have their entries set to that).  Receives q_start (int32 [n + 1]: where
        each sequence's new tokens begin among all), slots (int64, any size: a slot a new token, -1 behind the last), lens_out
        (may be lens) and n_free_out (may be n_free).  A sequence that there is no room for stays as it was, its slots -1."""
        dev, at = self.device, _dense_pointer
        (n,), (_, width) = _sizes(lens, "lens", 1), _sizes(block_table, "block_table", 2)
        (room,), (tokens,) = _sizes(free_blocks, "free_blocks", 1), _sizes(slots, "slots", 1)
        one, seqs = (1,), (n,)
        p = _b._Extend(at(lens, "lens", seqs, "int32", dev), at(add, "add", seqs, "int32", dev), at(block_table, "block_table", (n, width), "int32", dev),
                       at(free_blocks, "free_blocks", (room,), "int32", dev), at(n_free, "n_free", one, "int32", dev),
                       at(q_start, "q_start", (n + 1,), "int32", dev), at(slots, "slots", (tokens,), "int64", dev),
                       at(lens_out, "lens_out", seqs, "int32", dev), at(n_free_out, "n_free_out", one, "int32", dev), n, width, room, tokens, 0, 0)
        _check(self._calls.emoe_kv_extend(self._ref, ctypes.byref(p), _stream_handle(stream)))

    def keep(self, block_table, lens, q_start, accepted, n_accepted, change, stream=None, slots=None) -> None:
        """Moves the accepted nodes (int32 [n, most], rising node numbers, the first n_accepted [n] of each row) of the
        sequences' trees, their last q_start[s + 1] - q_start[s] tokens, to the front of these, in all layers.  change
        (int32 [n]) receives accepted less drafted tokens: the add of the next extend.  slots: those of the extend that took the
        nodes in; a sequence that was refused there, which has no nodes, stays as it is then (change 0)."""
        dev, at = self.device, _dense_pointer
        (n,), (_, width), (_, most) = _sizes(lens, "lens", 1), _sizes(block_table, "block_table", 2), _sizes(accepted, "accepted", 2)
        places = None if slots is None else at(slots, "slots", (_sizes(slots, "slots", 1)[0],), "int64", dev) or 8   # (an empty one has no address, and is not read)
        p = _b._Keep(at(block_table, "block_table", (n, width), "int32", dev), at(lens, "lens", (n,), "int32", dev),
                     at(q_start, "q_start", (n + 1,), "int32", dev), at(accepted, "accepted", (n, most), "int32", dev),
                     at(n_accepted, "n_accepted", (n,), "int32", dev), at(change, "change", (n,), "int32", dev), n, width, most, 0,
                     places, 0 if slots is None else slots.shape[0], 0)
        _check(self._calls.emoe_kv_keep(self._ref, ctypes.byref(p), _stream_handle(stream)))

    def attend_tree_workspace_bytes(self, n_seqs: int, n_tokens: int, max_q: int, n_q_heads: int, max_blocks: int) -> int:
        """Enough for calls of up to these sizes on this cache."""
        n = ctypes.c_uint64()
        _check(_b.lib().emoe_kv_attend_tree_workspace(self._ref, n_seqs, n_tokens, max_q, n_q_heads, max_blocks, ctypes.byref(n)))
        return n.value

    def attend_window_workspace_bytes(self, n_seqs: int, n_tokens: int, max_q: int, n_q_heads: int, max_blocks: int, window: int,
                                      sinks: int = 0) -> int:
        """Enough for calls of up to these sizes on this cache."""
        n = ctypes.c_uint64()
        _check(_b.lib().emoe_kv_attend_window_workspace(self._ref, n_seqs, n_tokens, max_q, n_q_heads, max_blocks, min(window, 1 << 30),
                                                        min(sinks, 1 << 30), ctypes.byref(n)))
        return n.value

    def attend_tree(self, layer: int, q, out, block_table, own_lens, q_start, mask, max_q: int, scale: Optional[float] = None, lse=None,
                    workspace=None, stream=None, wait_limit_us: int = 0) -> None:
        """Attention of trees of drafted tokens: q, out [n_tokens, n_q_heads, head_dim] (any stride between tokens), the
        nodes of sequence s at q_start[s] (int32 [n_seqs + 1]), at most max_q of them: the last ones of its own_lens[s] tokens.
        A node sees all tokens before the nodes and those nodes whose bits its row of mask (int32 [n_tokens, words]) has.
        workspace, lse, wait_limit_us: as for attend."""
        words = _sizes(mask, "mask", 2)[1]
        bits = _dense_pointer(mask, "mask", (q.shape[0], words), "int32", self.device)
        self._attend_rows(self._calls.emoe_kv_attend_tree, layer, q, out, block_table, own_lens, q_start, bits, max_q, words, 0, 0,
                          scale, lse, workspace, stream, wait_limit_us)

    def attend_window(self, layer: int, q, out, block_table, own_lens, q_start, max_q: int, window: int, sinks: int = 0,
                      scale: Optional[float] = None, lse=None, workspace=None, stream=None, wait_limit_us: int = 0) -> None:
        """Attention with a window: q, out and q_start as for attend_tree (single tokens and pieces of prompts, packed); a query
        token sees the last `window` tokens up to itself and the sequence's first `sinks` tokens."""
        self._attend_rows(self._calls.emoe_kv_attend_window, layer, q, out, block_table, own_lens, q_start, None, max_q, 0, min(window, 1 << 30),
                          min(sinks, 1 << 30), scale, lse, workspace, stream, wait_limit_us)

    def _attend_rows(self, call, layer, q, out, block_table, own_lens, q_start, mask, max_q, words, window, sinks, scale, lse, workspace, stream,
                     wait_limit_us):
        dev, at = self.device, _dense_pointer
        t, hq, hd = q.shape
        shape, row = (t, hq, self.head_dim), hq * self.head_dim
        if out.dtype != q.dtype:
            raise ValueError("out is %s, q %s" % (out.dtype, q.dtype))
        strides = [row, row]
        for i, (x, what) in enumerate(((q, "q"), (out, "out"))):
            if x.shape != shape or x.device != dev:
                _shaped(x, what, shape, None, dev)
            if not x.is_contiguous():
                _dense(x, what, 2)
                strides[i] = x.stride(0) if t > 1 else row
        (n,), (_, width) = _sizes(own_lens, "own_lens", 1), _sizes(block_table, "block_table", 2)
        work, size = _workspace(workspace, dev)
        p = _b._AttendRows(q.data_ptr(), out.data_ptr(), None if lse is None else at(lse, "lse", (t, hq), "float32", dev), strides[0], strides[1],
                           at(block_table, "block_table", (n, width), "int32", dev), at(own_lens, "own_lens", (n,), "int32", dev),
                           at(q_start, "q_start", (n + 1,), "int32", dev), mask, work, size, n, t, max_q, hq, width, words, window, sinks, _value_type(q, "q"),
                           hd ** -0.5 if scale is None else scale, wait_limit_us, 0)
        _check(call(self._ref, layer, ctypes.byref(p), _stream_handle(stream)))


class ExpertArena:
    """One rank's expert arena: emoe_moe_decode.

    arena: tensor or device address, [n_layers][3 (gate, up, down)][n_slots][matrix] as
    emoe_reshard_experts lays it out (or fused_w13), gate and up [d_ff, d_model], down [d_model, d_ff].
    w_type: "bf16", "f16" or "e4m3"; the last with fp32 scales per 128 x 128 block behind the weights, as
    a plan with expert_scale_bytes moves them.  matrix_stride: bytes from matrix to matrix in the paged
    stores (slab_bytes), 0 for a dense arena."""

    def __init__(self, arena, *, n_layers: int, n_slots: int, d_model: int, d_ff: int, w_type: str = "bf16",
                 fused_w13: bool = False, matrix_stride: int = 0, status=None):
        self._c = _b._ExpertArena(None, None, matrix_stride, n_layers, n_slots, d_model, d_ff, _type_of(w_type),
                                  _b.LAYOUT_FUSED_W13 if fused_w13 else 0, 0)
        self.w_type, self.d_model, self.d_ff, self.n_slots = self._c.type, d_model, d_ff, n_slots
        self._c.arena, self.device = _arena_pointer(arena, self.bytes(), "arena")
        if status is not None:
            self.device = self.device or status.device
            self._c.status = _shaped(status, "status", (1,), "int32", self.device).data_ptr()
        self._keep = (arena, status)
        self._ref = ctypes.byref(self._c)
        self._decode = _b.lib().emoe_moe_decode

    @classmethod
    def for_rank(cls, shape, n_slots: int, arena, w_type: str = "bf16", **kw) -> "ExpertArena":
        """The arena of a rank with n_slots slots of a model `shape`, as a plan with that shape lays it out."""
        if _TYPE_BYTES[_type_of(w_type)] != shape.elem_bytes:
            raise ValueError("%s elements have %d bytes, the shape's %d" % (w_type, _TYPE_BYTES[_type_of(w_type)], shape.elem_bytes))
        return cls(arena, n_layers=shape.n_layers, n_slots=n_slots, d_model=shape.d_model, d_ff=shape.d_ff, w_type=w_type, **kw)

    def bytes(self) -> int:
        n = ctypes.c_uint64()
        _check(_b.lib().emoe_expert_arena_bytes(ctypes.byref(self._c), ctypes.byref(n)))
        return n.value

    def decode_workspace_bytes(self, n_tokens: int, top_k: int, n_experts: int, n_shared: int = 0) -> int:
        """Enough for calls of up to these sizes."""
        n = ctypes.c_uint64()
        _check(_b.lib().emoe_moe_decode_workspace(self._ref, n_tokens, top_k, n_experts, n_shared, ctypes.byref(n)))
        return n.value

    def decode(self, layer: int, x, logits, top_k: int, slot_of_expert, out, n_shared: int = 0, renormalize: bool = True,
               routed_scale: float = 1.0, ids_out=None, weights_out=None, workspace=None, stream=None) -> None:
        """The layer for up to 64 tokens: x [n, d_model], logits float32 [n, n_experts], slot_of_expert int32
        [n_experts + n_shared] (-1: not in this arena), out [n, d_model] of x's type or float32 (a rank's
        part of the sum).  ids_out int32 / weights_out float32 [n, top_k] receive the choice.  workspace:
        decode_workspace_bytes bytes of the caller's, not shared by calls that can overlap."""
        n, experts = logits.shape
        _dense(_shaped(x, "x", (n, self.d_model), None, self.device), "x", 1)
        _dense(_shaped(logits, "logits", (n, experts), "float32", self.device), "logits", 1)
        _dense(_shaped(slot_of_expert, "slot_of_expert", (experts + n_shared,), "int32", self.device), "slot_of_expert", 1)
        _dense(_shaped(out, "out", (n, self.d_model), None, self.device), "out", 1)
        for t, what, dtype in ((ids_out, "ids_out", "int32"), (weights_out, "weights_out", "float32")):
            if t is not None:
                _dense(_shaped(t, what, (n, top_k), dtype, self.device), what, 2)
        p = _b._Moe(x.data_ptr(), logits.data_ptr(), slot_of_expert.data_ptr(), out.data_ptr(),
                    None if ids_out is None else ids_out.data_ptr(), None if weights_out is None else weights_out.data_ptr(),
                    *_workspace(workspace, self.device),
                    x.stride(0), logits.stride(0), out.stride(0), n, experts, n_shared, top_k,
                    _value_type(x, "x"), _value_type(out, "out"), 1 if renormalize else 0, routed_scale, 0)
        _check(self._decode(self._ref, layer, ctypes.byref(p), _stream_handle(stream)))
