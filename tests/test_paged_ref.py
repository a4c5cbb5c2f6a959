"""The plain implementations of the paged cache's calls against hand-worked values and against the contiguous ones (CPU only)."""
import math

import numpy as np
import pytest

import attention_ref as ref
import paged_ref as paged


def test_blocks_of_4_bits_by_hand():
    # the largest magnitude in units of the block's power of two is in [3.5, 7): 7 would round past 6 and takes twice the unit
    for top, unit in ((6.0, 1.0), (4.0, 1.0), (6.9999, 1.0), (7.0, 2.0), (8.0, 2.0), (3.9999, 1.0), (3.5, 1.0), (3.4999, 0.5), (1.0, 0.25), (2.0 ** -130, 2.0 ** -126)):
        assert paged.block_byte(top) == 127 + math.log2(unit), top
    assert paged.block_byte(0.0) == 1
    got = paged.nearest([0.0, 0.25, 0.2501, 0.75, 0.7499, 1.25, 1.75, 1.7499, 2.5, 2.5001, 3.5, 3.4999, 5.0, 5.0001, 6.9])
    assert got.tolist() == [0, 0, 1, 2, 1, 2, 4, 3, 4, 5, 6, 5, 6, 7, 7]
    # every tie goes to the even one of two codes
    assert all(c % 2 == 0 for c in paged.nearest(paged.TIES))


def test_blocks_hold_every_value_to_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 64)) * 10.0 ** rng.uniform(-30, 30, (50, 1))
    code, byte = paged.quantise(x)
    y = paged.values(code, byte)
    unit = np.repeat(2.0 ** (byte - 127.0), 32, -1)
    m = np.abs(x) / unit
    step = np.where(m <= 2, 0.5, np.where(m <= 4, 1.0, 2.0))
    assert np.all(np.abs(y - x) / unit <= step / 2) and np.all(np.abs(y) / unit <= 6)
    assert np.array_equal(paged.unpack(paged.pack(code)), code)
    again = paged.quantise(y)
    assert np.array_equal(paged.values(*again), y)             # what a block stands for is stored as it is
    x[0, 3], x[1, 40] = np.nan, np.inf
    byte = paged.quantise(x)[1]
    assert byte[0].tolist()[0] == 255 and byte[1].tolist()[1] == 255 and byte[0, 1] != 255 and byte[1, 0] != 255


def test_pages_in_order_are_a_contiguous_cache():
    rng = np.random.default_rng(2)
    B, T, Hq, H, d, page, n = 2, 5, 4, 2, 8, 16, 37
    q, k, v = rng.standard_normal((B, T, Hq, d)), rng.standard_normal((B, H, 48, d)), rng.standard_normal((B, H, 48, d))
    pool = lambda x: x.reshape(B, H, 3, page, d).transpose(0, 2, 1, 3, 4).reshape(B * 3, H, page, d)
    for window in (0, 6):
        a = paged.paged_attn(q, pool(k), pool(v), [[0, 1, 2], [3, 4, 5]], page, [n, 3], [T, 3], 0.3, window)
        w = ref.window_attn(q, k, v, [n, 3], [T, 3], window, 0, 0.3)
        for key in ("out", "lse", "mag", "n"):
            assert np.allclose(a[key], w[key], atol=1e-13)


@pytest.mark.parametrize("pos,length,kw,want", [
    (4, 10, {}, (0, 5)), (4, 10, dict(window=3), (2, 5)), (4, 10, dict(prefix=7), (0, 7)), (4, 10, dict(prefix=30), (0, 10)), (4, 10, dict(prefix=2), (0, 5)),
    (4, 10, dict(first=3), (3, 5)), (4, 10, dict(first=5), (0, 0)), (4, 10, dict(window=2, prefix=8, first=1), (3, 8)), (0, 1, dict(window=1), (0, 1))])
def test_sight(pos, length, kw, want):
    assert paged.span(pos, length, **kw) == want


def test_forms_of_scores():
    """Softmax over three keys by hand: capped, and with a slope."""
    k = np.array([1.0, 2.0, 4.0]).reshape(1, 1, 3, 1)
    k = np.concatenate([k, np.full((1, 1, 13, 1), np.nan)], 2)
    v = np.concatenate([np.array([1.0, 10.0, 100.0]).reshape(1, 1, 3, 1), np.full((1, 1, 13, 1), np.nan)], 2)
    one = lambda **kw: paged.paged_attn(np.ones((1, 1, 1, 1)), k, v, [[0]], 16, [3], [1], 1.0, **kw)
    x = 2 * np.tanh(np.array([1.0, 2.0, 4.0]) / 2) - 0.25 * np.array([2, 1, 0])
    w = np.exp(x) / np.exp(x).sum()
    r = one(cap=2.0, slopes=[0.25])
    assert np.isclose(r["out"][0, 0, 0, 0], w @ [1, 10, 100]) and np.isclose(r["lse"][0, 0, 0], np.log(np.exp(x).sum()))
    assert one(first=[[3]])["lse"][0, 0, 0] == -math.inf and np.all(one(first=[[3]])["out"] == 0)
