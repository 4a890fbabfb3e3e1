"""Plain 64-bit implementations of the serving operators on numpy arrays, and the layouts they work
on, written with numpy indexing only.  Test infrastructure."""
from __future__ import annotations

import numpy as np

TYPE_BYTES = {"bf16": 2, "f16": 2, "e4m3": 1}


def e4m3_values():
    """The value of each of the 256 codes (127 and 255 are NaN)."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = (-v if c & 128 else v) if (c & 127) != 127 else np.nan
    return out


E4M3 = e4m3_values()


def quantise(x):
    """(codes as values, scale bytes) of vectors along the last axis."""
    x = np.asarray(x, np.float64)
    flat = x.reshape(-1, x.shape[-1])
    codes, bytes_ = np.zeros_like(flat), np.zeros(len(flat), np.uint8)
    grid = np.sort(E4M3[:127])       # the non-negative values, ascending: code order
    for i, v in enumerate(flat):
        a = np.max(np.abs(v))
        if not np.isfinite(a):
            bytes_[i] = 255
            continue
        k = 0
        if a > 0:
            k = -126
            while a > 448 * 2.0 ** k:
                k += 1
        bytes_[i] = k + 127
        y = np.abs(v) / 2.0 ** k
        hi = np.clip(np.searchsorted(grid, y), 0, 126)
        lo = np.clip(hi - 1, 0, 126)
        dh, dl = np.abs(grid[hi] - y), np.abs(y - grid[lo])
        pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)   # to nearest, ties to the even code
        codes[i] = np.copysign(grid[pick], v)
    return codes.reshape(x.shape), bytes_.reshape(x.shape[:-1])


def scale_value(byte):
    byte = np.asarray(byte)
    return np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))


class Cache:
    """A logical cache: values [n_layers, 2, num_blocks, block_tokens, n_heads, head_dim] in 64 bits
    (for e4m3 the codes' values, with scale bytes beside them)."""

    def __init__(self, n_layers, num_blocks, block_tokens, n_heads, head_dim, kv_type, head_major=False):
        self.dims = (n_layers, 2, num_blocks, block_tokens, n_heads)
        self.head_dim, self.kv_type, self.head_major = head_dim, kv_type, head_major
        self.values = np.zeros(self.dims + (head_dim,))
        self.bytes = np.full(self.dims, 127, np.uint8)

    def order(self, x):
        """Logical order -> the order in memory."""
        return np.ascontiguousarray(x.swapaxes(3, 4)) if self.head_major else x

    def read(self, layer, kv, slot):
        """[heads, head_dim] of a token slot."""
        b, o = divmod(int(slot), self.dims[3])
        x = self.values[layer, kv, b, o]
        return x * scale_value(self.bytes[layer, kv, b, o])[:, None] if self.kv_type == "e4m3" else x


def attend(cache, layer, q, table, own_lens, prefix_table, prefix_len, scale):
    """q [n, t, Hq, hd] -> (o, lse, a, e) in 64 bits; tokens on blocks outside the pool are left out.
    a = sum_j softmax_j |v_j| and e = bound of a score's error for the tolerance: a sum of hd products
    in 32 bits is off by at most hd * 2^-23 (truncating adders) of the sum of their magnitudes, the sums
    over n tokens by n * 2^-23 of theirs, and the exponential adds a few 2^-22."""
    n, t, hq, hd = q.shape
    heads, block = cache.dims[4], cache.dims[3]
    group = hq // heads
    o, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    a, err = np.zeros(q.shape), np.zeros(q.shape[:3])

    def rows(ids, count):
        ks, vs = [], []
        for j in range(count):
            b = int(ids[j // block])
            if 0 <= b < cache.dims[2]:
                ks.append(cache.read(layer, 0, b * block + j % block))
                vs.append(cache.read(layer, 1, b * block + j % block))
        shape = (0, heads, hd)
        return (np.stack(ks) if ks else np.zeros(shape)), (np.stack(vs) if vs else np.zeros(shape))

    pk, pv = rows(prefix_table, prefix_len)
    for s in range(n):
        length = int(min(max(own_lens[s], 0), table.shape[1] * block))
        for i in range(t):
            ok, ov = rows(table[s], max(0, length - t + i + 1))
            k, v = np.concatenate([pk, ok]), np.concatenate([pv, ov])
            if not len(k):
                continue
            for h in range(hq):
                score = scale * (k[:, h // group] @ q[s, i, h])
                top = score.max()
                w = np.exp(score - top)
                lse[s, i, h] = top + np.log(w.sum())
                o[s, i, h] = (w / w.sum()) @ v[:, h // group]
                a[s, i, h] = (w / w.sum()) @ np.abs(v[:, h // group])
                size = np.abs(scale) * (np.abs(k[:, h // group]) @ np.abs(q[s, i, h])).max()
                err[s, i, h] = (hd + 8) * 2.0 ** -23 * size + (len(k) + 16) * 2.0 ** -23
    return o, lse, a, err


def route(logits, k):
    """(ids [T, k], softmax probabilities [T, k]) by (logit descending, id ascending); -1 / 0 where
    nothing above minus infinity is left; NaN counts as minus infinity."""
    logits = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    ids, p = np.full((len(logits), k), -1), np.zeros((len(logits), k))
    for t, row in enumerate(logits):
        order = sorted((e for e in range(len(row)) if row[e] > -np.inf), key=lambda e: (-row[e], e))[:k]
        if not order:
            continue
        top = row[order[0]]
        total = np.exp(row - top).sum()
        for i, e in enumerate(order):
            ids[t, i], p[t, i] = e, np.exp(row[e] - top) / total
    return ids, p
