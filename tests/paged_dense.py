"""paged_ref.paged_attn for one sequence of many queries, whole heads at a time, so that long prompts can be compared too."""
import math

import numpy as np

import paged_ref as paged
from attention_ref import U32


def paged_attn(q, k, v, table, page, n, scale, window=0, cap=0.0, slopes=None, fp32=False):
    """q [1][T][Hq][d] at the last T of n positions; k and v [pages][H][page][d] (float64), every page of `table` there: paged_ref's dict."""
    _, T, Hq, d = q.shape
    H = k.shape[1]
    r = dict(out=np.zeros(q.shape), lse=np.zeros(q.shape[:3]), mag=np.zeros(q.shape), S=np.zeros(q.shape[:3]), n=np.zeros(q.shape[:3], int))
    rows = lambda x, g: x[np.asarray(table), g].reshape(-1, d)[:n]
    pos, p = np.arange(n - T, n)[:, None], np.arange(n)
    low, high = np.array([paged.span(int(x), n, window) for x in pos[:, 0]]).T[..., None]
    seen = (p >= low) & (p < high)
    for h in range(Hq):
        K, V = rows(k, h // (Hq // H)), rows(v, h // (Hq // H))
        x = scale * (q[0, :, h] @ K.T)
        S = np.where(seen, np.abs(q[0, :, h]) @ np.abs(K).T, 0.0).max(-1) * abs(scale)
        extra = np.zeros(T)
        if cap:
            x = cap * np.tanh(x / cap)
            extra += 12 * U32 * (np.minimum(S, cap) if fp32 else cap)
        if slopes is not None:
            far = slopes[h] * np.abs(pos - p)
            x = x - far
            extra += 5 * U32 * np.where(seen, np.abs(far), 0.0).max(-1) + U32 * S
        x = np.where(seen, x, -math.inf)
        m = x.max(-1, keepdims=True)
        e = np.exp(x - m)
        w = e / e.sum(-1, keepdims=True)
        r["out"][0, :, h], r["mag"][0, :, h] = w @ V, w @ np.abs(V)
        r["lse"][0, :, h] = m[:, 0] + np.log(e.sum(-1))
        r["S"][0, :, h] = S + extra / ((d + 4) * U32)
        r["n"][0, :, h] = seen.sum(-1)
    return r
