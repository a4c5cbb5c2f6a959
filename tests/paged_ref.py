"""Plain 64-bit implementations of the paged cache's calls, and how far a kernel may be from them.

Rows of 4 bits: a block of 32 values is held exactly as its codes and its power of two say; storing rounds each value to the nearest code
(ties to the even one) under the power of two that the block's largest magnitude asks for.

Scores of clada_paged_attn add to attention_ref's score error e (u = 2^-24):
* cap tanh(x / cap) passes an error of x on undiminished at most.  In bf16 and 4-bit calls it is cap - 2 cap r, r = 1 / (1 + E), E = exp(2 x / cap): the
  argument's two roundings move r by r (1 - r) |ln E| 2 u <= 0.45 u, the exponential's 2 u by r (1 - r) 2 u <= u / 2, the sum's rounding and the
  reciprocal's 2 u by 3 u r; times 2 cap, with the roundings of cap and of the result: below 12 u cap.  In fp32 calls tanhf (2 u of its value
  at most, taken as 4), the products' roundings and the argument's: below 12 u min(|x|, cap).
* slopes |pos - p|: the slope's two roundings and the sum's, at most 3 u of it and u |x|, taken as 5 u (slope |pos - p|) + u |x|; |x| <= S.
These are added to S by the factor that turns S into e, (d + 4) u, so attention_ref.check bounds the output."""
import math

import numpy as np

import attention_ref as ref

U32 = ref.U32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TIES = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])       # between neighbours; the even code of two is the upper one at every second


def block_byte(top):
    """Exponent byte of a block whose largest magnitude is top (finite, not negative)."""
    if top == 0.0:
        return 1
    m, e = math.frexp(top)                                     # top = m 2^e, m in [1/2, 1)
    return min(max(e - 1 - 2 + (1 if m >= 0.875 else 0) + 127, 1), 252)      # 4 * 2^126 would be no finite fp32


def nearest(y):
    """Codes 0 to 7 of magnitudes in units of the block's power of two."""
    y = np.asarray(y, float)
    c = np.zeros(y.shape, int)
    for i, t in enumerate(TIES):
        c += (y >= t) if i % 2 else (y > t)
    return c


def quantise(x):
    """x [..., d] (float64) -> (codes [..., d] 0 to 15, bytes [..., d/32])."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(b).max(-1)
    byte = np.vectorize(lambda t: block_byte(t) if np.isfinite(t) else 255, otypes=[int])(top)
    unit = np.where(byte == 255, 1.0, 2.0 ** (byte - 127.0))[..., None]
    code = nearest(np.abs(np.where(np.isfinite(b), b, 0.0)) / unit) + 8 * (np.signbit(b) & (b == b))
    return code.reshape(x.shape), byte


def values(code, byte):
    """What codes [..., d] and bytes [..., d/32] stand for."""
    unit = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(float) - 127.0))
    v = np.where(code >= 8, -1.0, 1.0) * E2M1[code % 8]
    with np.errstate(over="ignore"):
        return v * np.repeat(unit, 32, -1)


def pack(code):
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def unpack(packed):
    p = packed.astype(int)
    return np.stack([p & 15, p >> 4], -1).reshape(*p.shape[:-1], -1)


def span(pos, length, window=0, prefix=None, first=None):
    """Keys [from, to) that a query at pos sees, pages aside."""
    end = pos + 1 if prefix is None else min(length, max(pos + 1, prefix))
    begin = max(0, pos - window + 1 if window else 0, 0 if first is None else first)
    return (begin, end) if begin < end else (0, 0)


def paged_attn(q, k, v, table, page, lens, q_lens, scale, window=0, cap=0.0, slopes=None, prefix=None, first=None, fp32=False):
    """q [B][T][Hq][d], k and v [pages][H][page][d] (float64), table [B][..]: attention_ref's dict, S with what the scores' forms add."""
    B, T, Hq, d = q.shape
    P, H = k.shape[:2]
    r = dict(out=np.zeros(q.shape), lse=np.full(q.shape[:3], -math.inf), mag=np.zeros(q.shape), S=np.zeros(q.shape[:3]), n=np.zeros(q.shape[:3], int))
    for b in range(B):
        for t in range(q_lens[b]):
            pos = lens[b] - q_lens[b] + t
            if pos < 0:
                continue
            lo, hi = span(pos, lens[b], window, None if prefix is None else prefix[b], None if first is None else first[b][t])
            p = np.array([x for x in range(lo, hi) if 0 <= table[b][x // page] < P], int)
            if not len(p):
                continue
            pages, rows = np.asarray(table[b])[p // page], p % page
            for h in range(Hq):
                g = h // (Hq // H)
                K, V = k[pages, g, rows], v[pages, g, rows]
                with np.errstate(invalid="ignore", over="ignore"):
                    x = scale * (K @ q[b, t, h])
                    S = float(np.max(np.abs(K) @ np.abs(q[b, t, h]))) * abs(scale)
                    extra = 0.0
                    if cap:
                        x = cap * np.tanh(x / cap)
                        extra += 12 * U32 * (min(S, cap) if fp32 else cap)
                    if slopes is not None:
                        far = slopes[h] * np.abs(pos - p)
                        x = x - far
                        extra += 5 * U32 * float(np.max(np.abs(far))) + U32 * S
                    m = x.max()
                    if m == -math.inf:                         # no score is above -inf
                        continue
                    e = np.exp(x - m)
                    w = e / e.sum()
                    r["out"][b, t, h], r["mag"][b, t, h] = w @ V, w @ np.abs(V)
                r["lse"][b, t, h] = m + np.log(e.sum())
                r["S"][b, t, h] = S + extra / ((d + 4) * U32)
                r["n"][b, t, h] = len(p)
    return r
