"""The paged cache's calls at the ends of what they accept: scales and caps near fp32's range, long prompts,
every exponent byte of 4-bit pages, wide rows, long pages."""
import math

import numpy as np
import pytest
import torch

import attention_ref as ref
import paged_dense as dense
import paged_ref as paged
from gpu_util import DEV, to_dev, to_np
from test_gpu_paged import TYPES, Pool, _case, _ints, _np_dtype, clada, ctx  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


# 64 (sequence, key head, 128 rows) units of 2000 keys: each is split in eight, so that a split has whole tiles between its first and its last one, which are
# taken by the loop without a look at single keys.
STEADY = dict(T=256, n=2000, H=16, Hq=32, page=64)


def _steady_pool(clada, kind, D, seed):
    pages = -(-STEADY["n"] // STEADY["page"])
    order = np.random.default_rng(seed).permutation(pages)
    return Pool(clada, kind, pages, STEADY["H"], STEADY["page"], D, order.reshape(1, -1), seed=seed), order


# A capped prompt's steady tiles take cap tanh(x / cap) as the product times a polynomial whose last coefficient holds cap log2(e) (scale / cap)^9: 3.8e38,
# 4e62 and 1e43 here, and 1e-44 and less in the last two.  The third number brings products of up to 6 to at most 0.4 of the cap, where the polynomial is taken.
GREAT = [(1e6, 4e9, 2.0 ** -16), (1e30, 4e33, 2.0 ** -16), (1e34, 1e35, 2.0 ** -8), (1e-12, 2.5e-16, 2.0 ** 8), (1e-35, 3e-39, 2.0 ** 8)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cap,scale,_", GREAT)
def test_prompts_whose_scale_over_cap_leaves_the_range(clada, ctx, kind, cap, scale, _):
    """Queries of zeros give scores of zero whatever the scale: the mean of the values, and the log of their number.  A weight of 1 is exact in bf16, a
    sum of n values is off by n 2^-24 of their magnitudes', the quotient and the last rounding follow."""
    T, n, D = STEADY["T"], STEADY["n"], 64
    pool, order = _steady_pool(clada, kind, D, 21)
    q = torch.zeros((1, T, STEADY["Hq"], D), dtype=pool.cache.dtype, device=DEV)
    out, lse = clada.paged_attn(ctx, q, pool.cache, _ints([n]), cap=cap, scale=scale, want_lse=True)
    v = pool.held("v")[order].transpose(1, 0, 2, 3).reshape(STEADY["H"], -1, D)
    unit = 2.0 ** -8 if kind != "f32" else 2.0 ** -24
    seen = np.arange(n - T + 1, n + 1)[:, None, None]
    want, mag = ((np.cumsum(x, 1)[:, n - T:n].transpose(1, 0, 2) / seen).repeat(2, 1) for x in (v, np.abs(v)))
    got, logs = to_np(out)[0], to_np(lse)[0]
    assert np.all(np.abs(got - want) <= unit * np.abs(want) + (seen + 16) * 2.0 ** -24 * mag)
    assert np.all(np.abs(logs - np.log(seen[..., 0])) <= (seen[..., 0] + 16) * 2.0 ** -24 + 4 * 2.0 ** -24 * np.log(seen[..., 0]))


def _one_of_many(clada, ctx, kind, T, n, cap, scale, q0=1.0, H=1):
    """Keys whose first value alone is not zero, one of 14 numbers from -6 to 6, times queries of q0: the largest score alone has a weight, as long as the next
    one differs from it by more than any exponent.  What came and what has to, and how far apart they may be: winners have one weight, which is off by
    one rounding to bf16 at most; their mean is a sum of at most n values."""
    D, page = 32, 16
    pages = -(-n // page)
    order = np.random.default_rng(3).permutation(pages * page)
    pool = Pool(clada, kind, pages, H, page, D, [list(range(pages))], seed=4)
    first = np.array([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])[order % 7] * np.where(order % 2, 1.0, -1.0)
    k = np.zeros((pages, H, page, D))
    k[..., 0] = first.reshape(pages, 1, page)
    k[..., 1] = 6.0                                            # (every block of 4 bits has the power 1; the queries' second value is 0)
    if kind == "mx4":
        code, byte = paged.quantise(k)
        pool.t["k"].copy_(torch.from_numpy(paged.pack(code)))
        pool.t["ks"].copy_(torch.from_numpy(byte.astype(np.uint8)))
    else:
        pool.t["k"].copy_(to_dev(k.astype(np.float32), kind))
    assert np.array_equal(pool.held("k"), k)
    q = torch.zeros((1, T, 2 * H, D), dtype=pool.cache.dtype, device=DEV)
    q[..., 0] = q0
    out, lse = clada.paged_attn(ctx, q, pool.cache, _ints([n]), cap=cap, scale=scale, want_lse=True)
    v = pool.held("v").transpose(1, 0, 2, 3).reshape(H, -1, D).repeat(2, 0)
    x = cap * np.tanh(first * q0 * scale / cap)
    want, mag, logs = np.zeros((T, 2 * H, D)), np.zeros((T, 2 * H, D)), np.zeros(T)
    for t in range(T):
        best = np.nonzero(x[:n - T + t + 1] == x[:n - T + t + 1].max())[0]
        want[t], mag[t] = v[:, best].mean(1), np.abs(v[:, best]).mean(1)
        logs[t] = x[best[0]] + math.log(len(best))
    unit, w = (2.0 ** -24, 0.0) if kind == "f32" else (2.0 ** -8, 2.0 ** -8 if T > 1 else 2.0 ** -16)
    assert np.all(np.abs(to_np(out)[0] - want) <= unit * np.abs(want) + ((n + 16) * 2.0 ** -24 + w) * mag)
    assert np.all(np.abs(to_np(lse)[0] - logs[:, None]) <= 16 * 2.0 ** -24 * cap + (n + 16) * 2.0 ** -24)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T,n,H", [(1, 90, 1), (STEADY["T"], STEADY["n"], STEADY["H"])])
@pytest.mark.parametrize("cap,scale,q0", GREAT[:3])
def test_small_products_of_great_scales(clada, ctx, kind, T, n, H, cap, scale, q0):
    """The largest product wins: it is ahead of the next one by 0.05 of the cap, a score is off by 12 2^-24 of the cap."""
    _one_of_many(clada, ctx, kind, T, n, cap, scale, q0, H)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T", [1, 100])
@pytest.mark.parametrize("cap,scale", [(2.3e38, 1e38), (1.5e38, 1e38), (2e38, -1e38), (1.2e38, 4e37), (8e37, 1e38), (1e30, 1e30)])
def test_caps_near_the_largest_number(clada, ctx, kind, T, cap, scale):
    """The same where twice the cap is beyond fp32; products of 4 and 6 differ by 9e-5 of the cap at least."""
    _one_of_many(clada, ctx, kind, T, T + 90, cap, scale)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("mods", [dict(), dict(cap=30.0), dict(cap=1.0), dict(cap=2.0, scale=-0.3), dict(bias=0.02), dict(cap=20.0, bias=0.5), dict(window=700, cap=5.0)],
                         ids=lambda m: "-".join(m) or "plain")
def test_steady_tiles(clada, ctx, kind, D, mods):
    """Long prompts: the loop without a look at single keys, capped below and above the polynomial's end, with slopes, behind a window."""
    T, n, Hq = STEADY["T"], STEADY["n"], STEADY["Hq"]
    pool, order = _steady_pool(clada, kind, D, D)
    rng = np.random.default_rng(D)
    q = to_dev(rng.standard_normal((1, T, Hq, D)), _np_dtype(kind))
    slopes = np.float32(rng.uniform(0.0, mods["bias"], Hq)) if "bias" in mods else None
    scale, window, cap = mods.get("scale", D ** -0.5), mods.get("window", 0), mods.get("cap", 0.0)
    out, lse = clada.paged_attn(ctx, q, pool.cache, _ints([n]), scale=scale, window=window, cap=cap, want_lse=True,
                                slopes=None if slopes is None else torch.from_numpy(slopes).to(DEV))
    r = dense.paged_attn(to_np(q), pool.held("k"), pool.held("v"), order, STEADY["page"], n, scale, window, cap, slopes, fp32=kind == "f32")
    ref.check(to_np(out), to_np(lse), r, _np_dtype(kind), weights_bf16=True)


# ------------------------------------------------------------------------------------------------ every exponent byte
def _every_byte(clada, table):
    """A pool of 16 pages of 16 rows, one head of 64 values: row b has the byte b and all 16 codes twice, then 255 - b and the codes backwards."""
    pool = Pool(clada, "mx4", 16, 1, 16, 64, table, seed=1)
    byte = np.stack([np.arange(256), 255 - np.arange(256)], -1)
    code = np.tile(np.concatenate([np.arange(32) % 16, 15 - np.arange(32) % 16]), (256, 1))
    want = paged.values(code, byte)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)      # beyond bf16
    for n in "kv":
        pool.t[n].copy_(torch.from_numpy(paged.pack(code).reshape(16, 1, 16, 32)))
        pool.t[n + "s"].copy_(torch.from_numpy(byte.astype(np.uint8).reshape(16, 1, 16, 2)))
    return pool, want


def test_every_byte_is_read(clada, ctx):
    """2^(byte - 127) from 0 on: values below the normal numbers are exact, those from 2^128 on infinite, and 255 is NaN for every code."""
    pool, want = _every_byte(clada, [list(range(16))])
    for x in clada.paged_read(ctx, pool.cache, _ints([list(range(256))])):
        got = to_np(x)[0, :, 0]
        bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
        assert not bad.any(), [(b, got[b][bad[b]][:4], want[b][bad[b]][:4]) for b in np.nonzero(bad.any(-1))[0][:4]]


@pytest.mark.parametrize("T", [1, 7, 40, 256])
def test_every_byte_as_a_value(clada, ctx, T):
    """A window of one: each query's output is the value that it sees, to the products' and the output's handling of numbers below 2^-126."""
    pool, want = _every_byte(clada, [list(range(16))])
    pool.t["k"].zero_()
    pool.t["ks"].fill_(127)
    q = to_dev(np.random.default_rng(2).standard_normal((1, T, 1, 64)), "bf16")
    for n in sorted({256, 255, 200, T}):
        if n < T:
            continue
        got, w = to_np(clada.paged_attn(ctx, q, pool.cache, _ints([n]), window=1))[0, :, 0], want[n - T:n]
        assert np.array_equal(np.isnan(got), np.isnan(w)), n
        near = np.abs(np.where(np.isfinite(w), got, 0.0) - np.where(np.isfinite(w), w, 0.0)) <= 2.0 ** -126
        assert np.all((got == w) | np.isnan(w) | (near & (np.abs(w) <= 2.0 ** -126))), n


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("byte,most,q", [(0, 7, 2.0 ** 126), (1, 7, 2.0 ** 125), (252, 7, 2.0 ** -126), (253, 5, 2.0 ** -126), (254, 3, 2.0 ** -126)])
def test_keys_at_both_ends_of_the_bytes(clada, ctx, byte, most, q, T):
    """Keys of the smallest and the largest powers of two, times queries that bring the scores back to units."""
    D, n = 64, T + 60
    pool = Pool(clada, "mx4", 8, 1, 16, D, [list(range(8))], seed=5)
    rng = np.random.default_rng(6)
    code = rng.integers(0, most + 1, (8, 1, 16, D)) + 8 * rng.integers(0, 2, (8, 1, 16, D))
    pool.t["k"].copy_(torch.from_numpy(paged.pack(code)))
    pool.t["ks"].fill_(byte)
    qs = to_dev(q * rng.choice([-1.0, 0.0, 0.0, 1.0], (1, T, 2, D)), "bf16")
    out, lse = clada.paged_attn(ctx, qs, pool.cache, _ints([n]), scale=0.5, want_lse=True)
    r = paged.paged_attn(to_np(qs), pool.held("k"), pool.held("v"), [list(range(8))], 16, [n], [T], 0.5)
    ref.check(to_np(out), to_np(lse), r, "bf16", weights_bf16=T > 1)


# ------------------------------------------------------------------------------------------------ sizes
@pytest.mark.parametrize("Hq,H", [(1, 1), (6, 2), (20, 1), (40, 1)])
def test_4_bit_heads_of_224(clada, ctx, Hq, H):
    """Seven blocks a row: a quarter of it, which a lane group takes, touches three of their exponents."""
    _case(clada, ctx, "mx4", 224, Hq, H, 1, [1, 0, 37, 300, 129], page=16, seed=Hq)
    _case(clada, ctx, "mx4", 224, Hq, H, 1, [300, 40, 33], page=64, seed=Hq + 1, heads_last=True, window=32, cap=3.0, bias=0.3)
    _case(clada, ctx, "mx4", 224, Hq, H, 9, [70, 9, 8], [9, 9, 8], page=16, seed=Hq + 2)
    _case(clada, ctx, "mx4", 224, Hq, H, 130, [207, 65], [130, 65], page=32, seed=Hq + 3, window=50, cap=4.0, bias=0.2)


@pytest.mark.parametrize("D", [160, 192, 224])
@pytest.mark.parametrize("page,heads_last", [(16, False), (256, True)])
def test_wide_4_bit_rows_are_read(clada, ctx, D, page, heads_last):
    pool = Pool(clada, "mx4", 3, 2, page, D, [[2, 0, -1]], seed=D, heads_last=heads_last)
    pos = [0, page - 1, page, 2 * page - 1, 2 * page, -1, 5]
    k, v = clada.paged_read(ctx, pool.cache, _ints([pos]))
    for got, n in ((k, "k"), (v, "v")):
        for t, p in enumerate(pos):
            want = pool.held(n)[[2, 0][p // page], :, p % page] if 0 <= p < 2 * page else np.zeros((2, D))
            assert np.array_equal(to_np(got)[0, t], want), (n, p)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("page", [256, 4096])
@pytest.mark.parametrize("T", [1, 7, 70])
def test_long_pages(clada, ctx, kind, page, T):
    """Pages of more rows than a tile, up to the longest: lengths that end on their border, one row around it and inside them."""
    _case(clada, ctx, kind, 32, 2, 1, T, [page + T, page, page + 1, 2 * page + 77], [T, T, min(T, 1), T], page=page, seed=T, cap=5.0)
    _case(clada, ctx, kind, 32, 2, 1, T, [2 * page + 5, page + 3], page=page, seed=T + 1, window=300, heads_last=True, holes=[(0, 1)])
