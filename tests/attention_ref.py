"""Plain 64-bit implementations of the cache and attention calls, and how far a kernel may be from them.

Rounding of an attention output, element by element (u = 2^-24 the unit of fp32's 24 significant bits, 2^-8 that of bf16's 8):

* a score is a sum of d products accumulated in fp32: off by at most e = (d + 4) u S, S = max_p scale sum_i |q_i k_pi| (the scaling's
  rounding among the 4); a weight p and the sum of weights are each off by a factor within exp(2 e) + 4 u (the exponential's own error);
* weights rounded to bf16 ahead of the product with the values (prompts) add 2^-8 of each weight, weights kept as two bf16 (16 bits)
  2^-16;
* the sum over n keys adds n u of sum_p p |v_p| at most, whatever its order;
* the output is rounded once: 2^-8 |o| in bf16, u |o| in fp32.

So |o - ref| <= unit |ref| + (4 e + (n + 16) u + w) sum_p p |v_p|, w the weights' unit, and |lse - ref| <= 2 e + (n + 16) u + 4 u |ref|."""
import math

import numpy as np

U32 = 2.0 ** -24


def cache_row(p, n_sink, ring):
    return p if ring == 0 or p < n_sink else n_sink + (p - n_sink) % ring


def attend(q, k, v, scale):
    """One query q [d] over keys k, v [n][d]: (o, lse, sum_p p |v_p|, S); nothing visible: zeros and -inf."""
    if len(k) == 0:
        return np.zeros(q.size), -math.inf, np.zeros(q.size), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * (k @ q)
        m = s.max()
        e = np.exp(s - m)
        lse = m + np.log(e.sum())
        p = e / e.sum()
        # a weight that is exactly zero takes part in the definition like any other
        return p @ v, lse, p @ np.abs(v), float(np.max(np.abs(k) @ np.abs(q))) * abs(scale)


def window_attn(q, kc, vc, lens, q_lens, window, sinks, scale, n_sink=0, ring=0):
    """q [B][T][Hq][d], kc, vc [B][H][cap][d] (float64): dict of out, lse, mag (sum p |v|), S, n (keys seen)."""
    B, T, Hq, d = q.shape
    H = kc.shape[1]
    r = dict(out=np.zeros(q.shape), lse=np.full(q.shape[:3], -math.inf), mag=np.zeros(q.shape), S=np.zeros(q.shape[:3]), n=np.zeros(q.shape[:3], int))
    for b in range(B):
        for t in range(q_lens[b]):
            pos = lens[b] - q_lens[b] + t
            seen = [p for p in range(pos + 1) if window == 0 or p > pos - window or p < sinks]
            rows = [cache_row(p, n_sink, ring) for p in seen]
            for h in range(Hq):
                g = h // (Hq // H)
                r["out"][b, t, h], r["lse"][b, t, h], r["mag"][b, t, h], r["S"][b, t, h] = attend(q[b, t, h], kc[b, g, rows], vc[b, g, rows], scale)
                r["n"][b, t, h] = len(rows)
    return r


def shared_prefix_attn(q, pk, pv, prefix_len, kc, vc, lens, scale):
    B, Hq, d = q.shape
    H = kc.shape[1]
    r = dict(out=np.zeros(q.shape), lse=np.zeros(q.shape[:2]), mag=np.zeros(q.shape), S=np.zeros(q.shape[:2]), n=np.zeros(q.shape[:2], int))
    for b in range(B):
        for h in range(Hq):
            g = h // (Hq // H)
            k = np.concatenate([pk[g, :prefix_len], kc[b, g, :lens[b]]])
            v = np.concatenate([pv[g, :prefix_len], vc[b, g, :lens[b]]])
            r["out"][b, h], r["lse"][b, h], r["mag"][b, h], r["S"][b, h] = attend(q[b, h], k, v, scale)
            r["n"][b, h] = len(k)
    return r


def check(out, lse, ref, dtype, weights_bf16=False):
    """out, lse (numpy float64) against a reference of the functions above, at the bound of this module."""
    d = out.shape[-1]
    e = (d + 4) * U32 * ref["S"]
    unit = 2.0 ** -8 if dtype == "bf16" else U32
    w = 0.0 if dtype == "f32" else 2.0 ** -8 if weights_bf16 else 2.0 ** -16
    fine = np.isfinite(ref["out"])
    assert np.array_equal(np.isfinite(out), fine), "values that are not finite in other places"
    rel = (4 * e + (ref["n"] + 16) * U32 + w)[..., None]
    with np.errstate(invalid="ignore"):
        off, bound = np.abs(out - ref["out"]), unit * np.abs(ref["out"]) + rel * ref["mag"]
    worst = np.max(np.where(fine, off - bound, -1.0), initial=-1.0)
    assert worst <= 1e-30, f"output off by {worst:.3e} more than the bound"
    if lse is not None:
        assert np.array_equal(np.isneginf(lse), np.isneginf(ref["lse"]))
        ok = np.isfinite(ref["lse"])
        assert np.array_equal(np.isfinite(lse), ok)
        off = np.abs(lse[ok] - ref["lse"][ok]) - (2 * e + (ref["n"] + 16) * U32)[ok] - 4 * U32 * np.abs(ref["lse"][ok])
        assert np.max(off, initial=-1.0) <= 0.0, f"lse off by {np.max(off):.3e} more than the bound"


def frequencies(R, theta=10000.0, kind="none", factor=8.0, original=4096.0, low=1.0, high=4.0):
    """(angles a position, magnitude) of the scalings, in 64 bits."""
    if kind == "base" and R > 2:
        theta = theta * factor ** (R / (R - 2))
    f = theta ** (-2.0 * np.arange(R // 2) / R)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "bands":
        s = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1)
        return (1 - s) * f / factor + s * f, 1.0
    if kind == "ramp":
        i = lambda n: R * math.log(original / (n * 2 * math.pi)) / (2 * math.log(theta))
        a, b = max(math.floor(i(high)), 0), min(math.ceil(i(low)), R - 1)
        g = np.clip((np.arange(R // 2) - a) / max(b - a, 0.001), 0, 1)
        return f / factor * g + f * (1 - g), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def rope(x, pos, f, layout, magnitude=1.0, weight=None, eps=None, offset=0.0):
    """x [B][T][H][d] (float64), pos [B][T]: norm and rotation; rows of a negative position are zeros."""
    x = x.copy()
    if eps is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * (weight + offset)
    R = 2 * len(f)
    a, b = (slice(0, R // 2), slice(R // 2, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
    ang = (pos[..., None].astype(np.float64) * f)[:, :, None]
    c, s = magnitude * np.cos(ang), magnitude * np.sin(ang)
    x[..., a], x[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    x[pos < 0] = 0.0
    return x
