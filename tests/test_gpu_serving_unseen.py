"""emoe_kv_attend: what a query token does not see has no influence on it, and what it sees is never dropped,
whatever the values are."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import serving_ref as R
from test_gpu_serving_attend import make_tables
from test_gpu_serving_kv import TORCH, device_cache, filled

pytestmark = pytest.mark.gpu


def call(c, q, table=None, lens=None, pt=None, prefix=0, scale=None):
    n, t, hq, _ = q.shape
    dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()    # noqa: E731
    out, lse = torch.empty_like(q), torch.empty(n, t, hq, device="cuda")
    work = torch.empty(c.attend_workspace_bytes(n, t, hq, 0 if table is None else table.shape[1], prefix), dtype=torch.uint8, device="cuda")
    c.attend(0, q, out, dev(table), dev(lens), dev(pt), prefix, scale=scale, lse=lse, workspace=work)
    return out, lse


@pytest.mark.parametrize("byte", [0, 141, 170, 200, 254])
@pytest.mark.parametrize("hd,group,t,io", [(64, 2, 2, "bf16"), (128, 4, 4, "f16"), (128, 8, 4, "bf16"), (256, 1, 3, "bf16"), (32, 5, 5, "f16")])
def test_scales_of_tokens_that_a_row_does_not_see(byte, hd, group, t, io):
    """The last own token's scales of an e4m3 cache may be any: the query tokens before it do not see it, so
    their outputs keep every bit."""
    rng = np.random.default_rng(hd + t)
    lens, prefix, block = [20, t, 33, 150, 64], 21, 16
    pool = 30
    ref = filled(rng, (1, pool, block, 2), hd, "e4m3", False)
    pt, table = make_tables(rng, pool, block, prefix, lens)
    clean = device_cache(ref)[0]
    c, _, scales = device_cache(ref)
    for s, n in enumerate(lens):
        scales[0, :, int(table[s, (n - 1) // block]), (n - 1) % block] = byte
    q = torch.from_numpy(rng.standard_normal((len(lens), t, 2 * group, hd))).to(TORCH[io]).cuda()
    for shared in (prefix, 0):
        want, got = (call(x, q, table, lens, pt if shared else None, shared) for x in (clean, c))
        assert torch.isfinite(want[0]).all()
        for x, y in zip(want, got):
            assert torch.equal(x[:, :-1], y[:, :-1])


@pytest.mark.parametrize("t", [1, 2])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_a_value_that_is_not_a_number_shows_whatever_its_weight(kv, t):
    """A token whose weight is below the smallest 32-bit number still has a part in the sum: a NaN in its value
    makes the row's output NaN, for 16-bit caches as for e4m3 ones."""
    ref = R.Cache(1, 6, 16, 2, 64, kv)
    ref.values[:, 0, 2, 5] = -2.0       # a score of -128 against 0: a weight of 2^-184
    ref.values[:, 1] = 1.0
    c, arena, scales = device_cache(ref)
    if kv == "e4m3":
        scales[0, 1, 2, 5, 0] = 255
    else:
        arena.view(torch.bfloat16).view(2, 6, 16, 2, 64)[1, 2, 5, 0] = float("nan")
    q = torch.ones(2, t, 4, 64, dtype=torch.bfloat16, device="cuda")
    table = np.array([[4, 2, 0], [1, 3, 5]], np.int32)
    out, lse = call(c, q, table, [40, 40], scale=1.0)
    assert torch.isnan(out[0, :, :2]).all()
    assert bool((out[0, :, 2:] == 1).all()) and bool((out[1] == 1).all())
    out, _ = call(c, q, pt=[0, 2], prefix=30, scale=1.0)
    assert torch.isnan(out[:, :, :2]).all() and bool((out[:, :, 2:] == 1).all())


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_a_value_that_is_not_a_number_in_a_split_of_no_weight(kv):
    """The same where all the tokens of its split have weights that small."""
    ref = R.Cache(1, 130, 16, 1, 64, kv)
    ref.values[:, 0, :64] = -2.0        # 1024 tokens
    ref.values[:, 1] = 1.0
    c, arena, scales = device_cache(ref)
    if kv == "e4m3":
        scales[0, 1, 0, 5, 0] = 255
    else:
        arena.view(torch.bfloat16).view(2, 130, 16, 1, 64)[1, 0, 5, 0] = float("nan")
    q = torch.ones(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    table = np.arange(130)[None]
    assert c.attend_workspace_bytes(1, 1, 2, 130, 0) > 0      # there are splits
    out, _ = call(c, q, table, [2000], scale=1.0)
    assert torch.isnan(out).all()
    out, _ = call(c, q, table[:, ::-1], [1000], scale=1.0)    # ends before it
    assert bool((out == 1).all())
    out, _ = call(c, q, pt=table[0], prefix=2000, scale=1.0)
    assert torch.isnan(out).all()


@pytest.mark.parametrize("rows,heads", [(4, 1), (33, 16)])
def test_tiny_queries_on_large_keys(rows, heads):
    """Queries of 2^-122 and e4m3 keys with scales of 2^117: their products are ordinary scores.  33 sequences on 16
    heads are work for the tensor core path (3 row tiles x 16 heads x 3200 tokens), 4 on one head for the other."""
    from test_gpu_serving_prefix_wide import definition
    rng = np.random.default_rng(11)
    prefix = 3200
    ref = R.Cache(1, 200, 16, heads, 128, "e4m3")
    codes = rng.integers(0, 127, ref.values.shape, dtype=np.uint8) | (rng.integers(0, 2, ref.values.shape, dtype=np.uint8) << 7)
    ref.values = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    ref.bytes[:, 0] = 127 + 117
    c, _, _ = device_cache(ref)
    pt = np.arange(200, dtype=np.int32)
    q = torch.from_numpy(rng.standard_normal((rows, 1, heads, 128)) * 2.0 ** -122).to(torch.bfloat16).cuda()
    assert float(q.abs().max()) > 2.0 ** -124
    out, lse = call(c, q, pt=pt, prefix=prefix)
    o, want, a, e = definition(ref, 0, q.double().cpu().numpy(), np.zeros((rows, 0), np.int32), [0] * rows, pt, prefix, 128 ** -0.5)
    assert want.std() > 0.01     # the scores matter
    # A query's power of two (2^127 at most) and the call's scale meet in a 32-bit factor of 2^-131 or more: off by
    # half its smallest step 2^-149, 2^-19 of a score.  Scores are at most |want| + log(tokens) from it.
    size = 2.0 ** -19 * (np.abs(want) + 2 * np.log(prefix) + 40)
    assert (np.abs(lse.double().cpu().numpy() - want) <= e + size + 2.0 ** -20).all()
    # weights and result rounded to 16 bits, scores off by that, weights below f16's normal range (2^-31 of v's largest
    # scale, 1 here, times the code)
    v = np.abs(ref.values[0, 1].reshape(-1, heads, 128)).sum(0)
    tol = 1.05 * (2 * 2.0 ** -8 + 2 * (e + size)[..., None]) * a + 2.0 ** -31 * v[None, None]
    assert (np.abs(out.double().cpu().numpy() - o) <= tol).all()


@pytest.mark.parametrize("rows,heads", [(4, 1), (33, 24)])
def test_values_far_below_the_16_bit_ones(rows, heads):
    """Values of 2^-24 and less in an e4m3 cache, with bf16 outputs, which reach as far: nothing is lost (24 heads x
    3 row tiles x 2000 tokens: the tensor core path)."""
    from test_gpu_serving_prefix_wide import definition, wide
    rng = np.random.default_rng(12)
    ref = wide(rng, (1, 125, 16, heads), 128, "e4m3")
    pt = np.arange(125, dtype=np.int32)
    q = torch.from_numpy(rng.standard_normal((rows, 1, heads, 128)) * 0.2).to(torch.bfloat16).cuda()
    for low, high in ((127 - 33, 127 - 33), (127 - 100, 127 - 100), (1, 1), (127 - 60, 127 - 33)):
        ref.bytes[:, 1] = rng.integers(low, high + 1, ref.bytes[:, 1].shape)
        c, _, _ = device_cache(ref)
        out, _ = call(c, q, pt=pt, prefix=2000)
        o, _, a, e = definition(ref, 0, q.double().cpu().numpy(), np.zeros((rows, 0), np.int32), [0] * rows, pt, 2000, 128 ** -0.5)
        v = np.abs(ref.values[0, 1].reshape(-1, heads, 128)).sum(0)
        top = 2.0 ** (int(ref.bytes[0, 1].max()) - 127)
        # bf16's own smallest step, 2^-133, beside the tolerance of the tests above
        tol = 1.05 * (2 * 2.0 ** -8 + 2 * e[..., None]) * a + 2.0 ** -31 * top * v[None, None] + 2.0 ** -134
        assert np.mean(np.abs(o) > tol) > 0.7      # an output of zeros would not pass
        assert (np.abs(out.double().cpu().numpy() - o) <= tol).all()
