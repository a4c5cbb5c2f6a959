"""clada_qk_rope against the plain 64-bit implementation (attention_ref.py).

Rounding: the norm's factor is off by a few units of 2^-24 (d terms in 16-byte pieces and a tree: d/4 + 8 at most), a cosine or sine by 2^-22
(the turn to 2^-25 of a turn, the function itself to 2^-23), the rotation by three roundings; the result is rounded once (unit 2^-8 in bf16, 2^-24 in
fp32).  So
|y - ref| <= unit |ref| + (d/4 + 24) 2^-24 (|x_a| + |x_b|) magnitude, x_a and x_b the normed pair."""
import numpy as np
import pytest
import torch

import attention_ref as ref
from gpu_util import DEV, to_dev, to_np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def clada():
    import paper_2502_19078_amd as pkg
    return pkg


@pytest.fixture(scope="module")
def ctx(clada):
    return clada.Context(0, 256)


def _draw(seed, dtype, *shape):
    return to_dev(np.random.default_rng(seed).standard_normal(shape), dtype)


def _check(got, x, pos, f, layout, magnitude, weight, eps, offset, dtype):
    want = ref.rope(x, pos, f, layout, magnitude, weight, eps, offset)
    plain = ref.rope(x, np.where(pos < 0, -1, 0), f, layout, 1.0, weight, eps, offset)
    R = 2 * len(f)
    pair = np.abs(plain)
    if R:
        a, b = (slice(0, R // 2), slice(R // 2, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
        both = (pair[..., a] + pair[..., b]) * max(abs(magnitude), 1.0)
        pair[..., a], pair[..., b] = both, both
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    bound = unit * np.abs(want) + (x.shape[-1] / 4 + 24) * 2.0 ** -24 * pair
    assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) - bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,R,layout", [(128, 128, "half"), (128, 64, "half"), (128, 128, "pairs"), (64, 64, "half"), (80, 32, "pairs"), (80, 80, "half"),
                                        (96, 24, "half"), (256, 256, "half"), (256, 2, "pairs"), (8, 8, "half"), (192, 192, "pairs"), (64, 0, "half"),
                                        (72, 18, "pairs"), (72, 36, "half")])
@pytest.mark.parametrize("norm", [False, True])
def test_rotation_and_norm(clada, ctx, dtype, D, R, layout, norm):
    B, T, Hq, H, cap = 2, 5, 6, 2, 40
    pos = np.array([[0, 1, 2, 3, 4], [30, 31, 32, -1, -1]], np.int32)
    f, mag = ref.frequencies(R) if R else (np.zeros(0), 1.0)
    plan = clada.rope_plan(ctx, R, layout=clada.ROPE_HALF if layout == "half" else clada.ROPE_PAIRS) if R else \
        clada.RopePlan(torch.empty(0, dtype=torch.int64, device=DEV))
    x = _draw(D + R, dtype, B, T, Hq + 2 * H, D)                # one projection's output: views with strides
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
    kc, vc = (torch.full((B, H, cap, D), 7.0, dtype=x.dtype, device=DEV) for _ in range(2))
    w = [_draw(90 + i, dtype, D) for i in range(2)] if norm else [None, None]
    kw = dict(q_norm=w[0], k_norm=w[1], eps=1e-5, norm_offset=1.0) if norm else {}
    out = clada.qk_rope(ctx, plan, q, k, v, torch.from_numpy(pos).to(DEV), clada.KVCache(kc, vc), **kw)
    args = (f, layout, mag)
    wn = [to_np(a) for a in w] if norm else [None, None]
    eps = 1e-5 if norm else None
    _check(to_np(out), to_np(q), pos, *args, wn[0], eps, 1.0, dtype)
    kr, vr, kn, vn = to_np(k), to_np(v), to_np(kc), to_np(vc)
    stored = np.zeros((B, cap), bool)
    for b in range(B):
        for t in range(T):
            if pos[b, t] >= 0:
                stored[b, pos[b, t]] = True
                _check(kn[b:b + 1, None, :, pos[b, t]], kr[b:b + 1, t:t + 1], pos[b:b + 1, t:t + 1], *args, wn[1], eps, 1.0, dtype)
                assert np.array_equal(vn[b, :, pos[b, t]], vr[b, t])
    for c in (kn, vn):                                          # nothing else is touched
        assert np.all(np.moveaxis(c, 2, 1)[~stored] == 7.0)


@pytest.mark.parametrize("kind", ["none", "linear", "base", "bands", "ramp"])
@pytest.mark.parametrize("R,theta", [(128, 500000.0), (64, 10000.0), (2, 10000.0)])
def test_scalings_and_far_positions(clada, ctx, kind, R, theta):
    """fp32 heads: at position 2^31 - 1 an angle formed in fp32 would be off by whole turns."""
    D = 128
    pos = np.array([[0, 1, 4095, 131071, 1 << 24, (1 << 24) + 1, 123456789, 2 ** 31 - 1]], np.int32)
    f, mag = ref.frequencies(R, theta, kind)
    code = ["none", "linear", "base", "bands", "ramp"].index(kind)
    plan = clada.rope_plan(ctx, R, theta, scaling=code, factor=8.0, original_len=4096.0, low=1.0, high=4.0)
    assert abs(plan.magnitude - mag) < 1e-6
    q = _draw(5, "f32", 1, 8, 3, D)
    kc = torch.zeros(1, 1, 1, D, device=DEV)
    out = clada.qk_rope(ctx, plan, q, None, None, torch.from_numpy(pos).to(DEV), clada.KVCache(kc, kc.clone()))
    # the frequencies themselves are 64-bit values: a relative 2^-50 of a far angle is 2^-19 of a radian
    want = ref.rope(to_np(q), pos, f, "half", mag)
    far = pos[0].astype(np.float64)[None, :, None, None] * f.max() * 2.0 ** -50
    x = np.abs(to_np(q))
    assert np.all(np.abs(to_np(out) - want) <= (56 * 2.0 ** -24 + far) * 2 * mag * x.max())


def test_in_place_ring_slots_and_one_side_alone(clada, ctx):
    D, H, B, T = 64, 3, 2, 4
    plan = clada.rope_plan(ctx, D)
    q, k, v = (_draw(i, "bf16", B, T, H, D) for i in range(3))
    pos = torch.tensor([[0, 1, 2, 3], [21, 22, 23, 24]], dtype=torch.int32, device=DEV)
    cache = lambda **kw: clada.KVCache(*(torch.zeros(B, 9, H, D, dtype=torch.bfloat16, device=DEV).transpose(1, 2) for _ in range(2)), **kw)
    c0 = cache(n_sink=2, ring=7)
    out = clada.qk_rope(ctx, plan, q, k, v, pos, c0)
    mine = q.clone()
    assert clada.qk_rope(ctx, plan, mine, None, None, pos, c0, out=mine) is mine and torch.equal(mine, out)
    rows = [[ref.cache_row(p, 2, 7) for p in r] for r in pos.tolist()]
    c1 = cache()
    slots = torch.tensor(rows, dtype=torch.int32, device=DEV)
    assert clada.qk_rope(ctx, plan, None, k, v, pos, c1, slots=slots) is None
    assert torch.equal(c0.k, c1.k) and torch.equal(c0.v, c1.v)
    for b in range(B):
        for t in range(T):
            assert torch.equal(c0.v[b, :, rows[b][t]], v[b, t])
    # rows outside the cache are not stored, by slot or by position
    c2 = cache()
    clada.qk_rope(ctx, plan, None, k, v, pos, c2, slots=torch.full_like(slots, -1))
    clada.qk_rope(ctx, plan, None, k, v, pos, c2, slots=torch.full_like(slots, 9))
    clada.qk_rope(ctx, plan, None, k[1:], v[1:], pos[1:].contiguous(), c2)
    assert not c2.k.any() and not c2.v.any()
    with pytest.raises(clada.CladaError):                       # more tokens than the ring holds
        clada.qk_rope(ctx, plan, None, _draw(1, "bf16", B, 8, H, D), _draw(2, "bf16", B, 8, H, D),
                      torch.zeros(B, 8, dtype=torch.int32, device=DEV), c0)


def test_a_norm_without_weights_and_weights_without_a_norm(clada, ctx):
    D = 64
    plan, pos = clada.rope_plan(ctx, D), torch.tensor([[5, 6]], dtype=torch.int32, device=DEV)
    cache = clada.KVCache(*(torch.zeros(1, 1, 8, D, device=DEV) for _ in range(2)))
    q, w = _draw(1, "f32", 1, 2, 3, D), _draw(2, "f32", D)
    f, _ = ref.frequencies(D)
    p = pos.cpu().numpy()
    _check(to_np(clada.qk_rope(ctx, plan, q, None, None, pos, cache, norm=True, eps=0.1)), to_np(q), p, f, "half", 1.0, None, 0.1, 0.0, "f32")
    _check(to_np(clada.qk_rope(ctx, plan, q, None, None, pos, cache, q_norm=w, norm=False)), to_np(q), p, f, "half", 1.0, None, None, 0.0, "f32")
    _check(to_np(clada.qk_rope(ctx, plan, q, None, None, pos, cache, k_norm=w, eps=0.1)), to_np(q), p, f, "half", 1.0, None, 0.1, 0.0, "f32")


@pytest.mark.parametrize("T", [1, 7, 600])
def test_many_tokens_and_heads(clada, ctx, T):
    """Every count of heads a group takes: few tokens spread over the chip, many share their angles."""
    B, Hq, H, D = 3, 32, 8, 128
    plan = clada.rope_plan(ctx, D)
    f, _ = ref.frequencies(D)
    q, k, v = (_draw(i, "bf16", B, T, h, D) for i, h in ((1, Hq), (2, H), (3, H)))
    pos = torch.arange(T, dtype=torch.int32, device=DEV).repeat(B, 1)
    kc, vc = (torch.zeros(B, T, H, D, dtype=torch.bfloat16, device=DEV).transpose(1, 2) for _ in range(2))
    out = clada.qk_rope(ctx, plan, q, k, v, pos, clada.KVCache(kc, vc))
    _check(to_np(out), to_np(q), pos.cpu().numpy(), f, "half", 1.0, None, None, 0.0, "bf16")
    _check(to_np(kc.transpose(1, 2)), to_np(k), pos.cpu().numpy(), f, "half", 1.0, None, None, 0.0, "bf16")
    assert torch.equal(vc.transpose(1, 2), v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_a_norm_of_values_whose_squares_are_subnormal(clada, ctx, dtype, layout):
    """eps = 0 and heads of +-2^-64: the mean square 2^-128 is exact and below fp32's normal numbers; the normed values are +-1."""
    D = 64
    plan = clada.rope_plan(ctx, D, layout=clada.ROPE_HALF if layout == "half" else clada.ROPE_PAIRS)
    pos = torch.tensor([[0, 3, 70]], dtype=torch.int32, device=DEV)
    cache = clada.KVCache(*(torch.zeros(1, 1, 1, D, dtype=_draw(1, dtype, 1).dtype, device=DEV) for _ in range(2)))
    q = torch.sign(_draw(1, dtype, 1, 3, 5, D)) * 2.0 ** -64
    w = _draw(2, dtype, D)
    f, _ = ref.frequencies(D)
    out = clada.qk_rope(ctx, plan, q, None, None, pos, cache, q_norm=w, eps=0.0)
    _check(to_np(out), to_np(q), pos.cpu().numpy(), f, layout, 1.0, to_np(w), 0.0, 0.0, dtype)
