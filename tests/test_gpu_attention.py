"""clada_window_attn and clada_shared_prefix_attn against the plain 64-bit implementation and its rounding bound (attention_ref.py)."""
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
    return clada.Context(0, clada.attn_workspace_bytes(64, 1024, 64, 256))


def _draw(rng, dtype, *shape):
    return to_dev(rng.standard_normal(shape), dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _window_case(clada, ctx, dtype, D, Hq, H, T, lens, q_lens, window, sinks, n_sink=0, ring=0, cap=None, seed=0, stale=float("nan"), heads_last=False):
    """Random queries and cache; rows that no position of the sequence lies in hold `stale`."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    cap = cap or (n_sink + ring if ring else max(max(lens), 1))
    shape = (B, cap, H, D) if heads_last else (B, H, cap, D)
    kc, vc = (_draw(rng, dtype, *shape) for _ in range(2))
    if heads_last:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    for b, n in enumerate(lens):
        held = torch.zeros(cap, dtype=torch.bool, device=DEV)
        held[[ref.cache_row(p, n_sink, ring) for p in range(n)]] = True
        kc[b, :, ~held] = stale
        vc[b, :, ~held] = stale
    q = _draw(rng, dtype, B, T, Hq, D)
    ql = q_lens if q_lens is not None else [T] * B
    for b in range(B):
        q[b, ql[b]:] = stale
    out, lse = clada.window_attn(ctx, q, clada.KVCache(kc, vc, n_sink, ring), _ints(lens), None if q_lens is None else _ints(q_lens), window, sinks,
                                 want_lse=True)
    r = ref.window_attn(to_np(q), to_np(kc), to_np(vc), lens, ql, window, sinks, D ** -0.5, n_sink, ring)
    ref.check(to_np(out), to_np(lse), r, dtype, weights_bf16=T > 1)
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [8, 64, 72, 80, 96, 128, 192, 256])
@pytest.mark.parametrize("Hq,H", [(1, 1), (6, 2), (8, 1), (20, 1), (40, 1)])
def test_single_token(clada, ctx, dtype, D, Hq, H):
    _window_case(clada, ctx, dtype, D, Hq, H, 1, [1, 0, 37, 300, 129], None, 0, 0, seed=D + Hq)
    _window_case(clada, ctx, dtype, D, Hq, H, 1, [300, 40, 33], None, 32, 4, cap=301, seed=D + Hq + 1, heads_last=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (7, 3), (40, 4), (64, 0), (500, 2), (16, 100)])
@pytest.mark.parametrize("T", [1, 2, 9, 33, 150])
def test_windows_and_sinks(clada, ctx, dtype, window, sinks, T):
    """Lengths shorter than the queries (positions below zero), equal (a prompt), longer (a chunk), zero; ragged queries, none among them."""
    _window_case(clada, ctx, dtype, 64, 4, 2, T, [T, T + 100, max(T - 1, 0), 0, T + 31], [T, T, T, T, max(T // 2, 0)], window, sinks, seed=T + window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,H", [(128, 4, 1), (80, 3, 3), (256, 5, 1), (96, 7, 1), (64, 2, 1), (40, 2, 2), (200, 2, 1)])
@pytest.mark.parametrize("T,extra", [(65, 0), (128, 1), (200, 77), (260, 0)])
def test_prompts(clada, ctx, dtype, D, Hq, H, T, extra):
    _window_case(clada, ctx, dtype, D, Hq, H, T, [T + extra, T // 2 + extra], [T, T // 2], 0, 0, seed=T + D)
    _window_case(clada, ctx, dtype, D, Hq, H, T, [T + extra, T // 3], [T, T // 3], 50, 3, seed=T + D + 1, heads_last=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,window,sinks,n_sink,ring", [(1, 32, 4, 4, 32), (1, 10, 0, 0, 10), (1, 33, 2, 5, 50), (9, 24, 4, 4, 32), (64, 40, 1, 3, 110), (20, 1, 0, 0, 20)])
def test_rings(clada, ctx, dtype, T, window, sinks, n_sink, ring):
    """The oldest positions have been written over; lengths before, at and behind each wrap."""
    for base in (0, n_sink, n_sink + ring - T, n_sink + ring, 3 * ring + 7, 1000003):
        n = max(base, 0) + T
        lens = [n, n + 1, n + ring // 2]
        rng = np.random.default_rng(n)
        q = _draw(rng, dtype, 3, T, 4, 64)
        kc, vc = (_draw(rng, dtype, 3, 2, n_sink + ring, 64) for _ in range(2))
        out, lse = clada.window_attn(ctx, q, clada.KVCache(kc, vc, n_sink, ring), _ints(lens), None, window, sinks, want_lse=True)
        # the reference over the positions that matter, moved down to where they are few
        K, V, Q = to_np(kc), to_np(vc), to_np(q)
        r = dict(out=np.zeros(Q.shape), lse=np.zeros(Q.shape[:3]), mag=np.zeros(Q.shape), S=np.zeros(Q.shape[:3]), n=np.zeros(Q.shape[:3], int))
        for b in range(3):
            for t in range(T):
                pos = lens[b] - T + t
                seen = sorted({p for p in range(max(pos - window + 1, 0), pos + 1)} | {p for p in range(min(sinks, pos + 1))})
                rows = [ref.cache_row(p, n_sink, ring) for p in seen]
                for h in range(4):
                    r["out"][b, t, h], r["lse"][b, t, h], r["mag"][b, t, h], r["S"][b, t, h] = ref.attend(Q[b, t, h], K[b, h // 2, rows], V[b, h // 2, rows], 0.125)
                    r["n"][b, t, h] = len(rows)
        ref.check(to_np(out), to_np(lse), r, dtype, weights_bf16=T > 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T,window", [(1, 8), (5, 0), (40, 8), (150, 60)])
def test_what_is_masked_does_not_reach_the_output(clada, ctx, dtype, bad, T, window):
    """A row of the cache that is not finite reaches the queries that see it and no others."""
    rng = np.random.default_rng(7)
    D, Hq, H, n = 64, 4, 2, T + 20
    q = _draw(rng, dtype, 1, T, Hq, D)
    kc, vc = (_draw(rng, dtype, 1, H, n, D) for _ in range(2))
    at = n - 1 - T // 3                                         # seen by the last third at most
    vc[0, :, at, 5] = bad
    vc[0, 1, at, 17] = bad
    out, lse = clada.window_attn(ctx, q, clada.KVCache(kc, vc), _ints([n]), None, window, 0, want_lse=True)
    clean = vc.clone()
    clean[0, :, at] = 0.0
    r = ref.window_attn(to_np(q), to_np(kc), to_np(clean), [n], [T], window, 0, D ** -0.5)
    sees = np.array([at <= n - T + t and (window == 0 or at > n - T + t - window) for t in range(T)])
    want = ref.window_attn(to_np(q), to_np(kc), to_np(vc), [n], [T], window, 0, D ** -0.5)
    got = to_np(out)
    assert np.array_equal(np.isnan(got), np.isnan(want["out"])) and np.array_equal(np.isposinf(got), np.isposinf(want["out"]))
    for t in np.nonzero(~sees)[0]:
        one = {k: v[:, t:t + 1] for k, v in r.items()}
        ref.check(got[:, t:t + 1], to_np(lse)[:, t:t + 1], one, dtype, weights_bf16=T > 1)
    # and a key that is not finite makes the scores of those queries so
    kc[0, 0, at] = bad
    out = to_np(clada.window_attn(ctx, q, clada.KVCache(kc, clean), _ints([n]), None, window, 0))
    assert np.all(np.isfinite(out[0, ~sees]))
    if bad != bad:
        assert np.all(np.isnan(out[0, sees][:, :Hq // H]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_a_lowest_value(clada, ctx, dtype):
    """Scores of thousands, and keys of the type's lowest value."""
    rng = np.random.default_rng(3)
    D, n = 64, 90
    q, kc, vc = _draw(rng, dtype, 1, 3, 2, D) * 40, _draw(rng, dtype, 1, 1, n, D) * 40, _draw(rng, dtype, 1, 1, n, D)
    out, lse = clada.window_attn(ctx, q, clada.KVCache(kc, vc), _ints([n]), None, 0, 0, want_lse=True)
    r = ref.window_attn(to_np(q), to_np(kc), to_np(vc), [n], [3], 0, 0, D ** -0.5)
    ref.check(to_np(out), to_np(lse), r, dtype, weights_bf16=True)
    q = q.abs() * 1e-3
    kc[0, 0, 10:20] = torch.finfo(kc.dtype).min / 1e3           # scores around -1e36: weights of exactly zero
    out = clada.window_attn(ctx, q, clada.KVCache(kc, vc), _ints([n]), None, 0, 0)
    keep = [p for p in range(n) if not 10 <= p < 20]
    r = ref.window_attn(to_np(q), to_np(kc)[:, :, keep], to_np(vc)[:, :, keep], [n - 10], [3], 0, 0, D ** -0.5)
    ref.check(to_np(out), None, r, dtype, weights_bf16=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,H,B", [(128, 8, 2, 3), (64, 4, 4, 1), (80, 5, 5, 17), (256, 8, 1, 5), (96, 6, 3, 40), (64, 40, 2, 2), (128, 16, 1, 64)])
@pytest.mark.parametrize("P", [1, 31, 500])
def test_shared_prefix(clada, ctx, dtype, D, Hq, H, B, P):
    rng = np.random.default_rng(D + B + P)
    q = _draw(rng, dtype, B, Hq, D)
    pk, pv = (_draw(rng, dtype, 1, H, P + 3, D) for _ in range(2))
    kc, vc = (_draw(rng, dtype, B, H, 40, D) for _ in range(2))
    lens = [int(v) for v in rng.integers(0, 41, B)]
    lens[0] = 0
    for c in (pk, pv):
        c[:, :, P:] = float("nan")
    for b, n in enumerate(lens):
        kc[b, :, n:] = float("nan")
        vc[b, :, n:] = float("nan")
    out, lse = clada.shared_prefix_attn(ctx, q, clada.KVCache(pk, pv), P, clada.KVCache(kc, vc), _ints(lens), want_lse=True)
    r = ref.shared_prefix_attn(to_np(q), to_np(pk)[0], to_np(pv)[0], P, to_np(kc), to_np(vc), lens, D ** -0.5)
    ref.check(to_np(out), to_np(lse), r, dtype, weights_bf16=True)


def test_strides_and_outputs_in_place_of_others(clada, ctx):
    """Queries and outputs as slices of wider tensors, the cache with rows of all heads side by side; nothing outside is written."""
    rng = np.random.default_rng(11)
    B, T, Hq, H, D, n = 2, 6, 4, 2, 64, 50
    wide = _draw(rng, "bf16", B, T, Hq + 2 * H, D)
    q = wide[:, :, :Hq]
    kc, vc = (_draw(rng, "bf16", B, n, 2 * H, D)[:, :, :H].transpose(1, 2) for _ in range(2))
    to = torch.full((B, T, Hq + 3, D), 9.0, dtype=torch.bfloat16, device=DEV)
    clada.window_attn(ctx, q, clada.KVCache(kc, vc), _ints([n, 30]), None, 20, 2, out=to[:, :, 1:Hq + 1])
    same = clada.window_attn(ctx, q.contiguous(), clada.KVCache(kc.contiguous(), vc.contiguous()), _ints([n, 30]), None, 20, 2)
    assert torch.equal(to[:, :, 1:Hq + 1], same)
    assert torch.all(to[:, :, 0] == 9.0) and torch.all(to[:, :, Hq + 1:] == 9.0)
    # scale, and a broadcast query
    one = q[:, :1].expand(B, T, Hq, D)
    a = clada.window_attn(ctx, one, clada.KVCache(kc, vc), _ints([n, 30]), None, 20, 2, scale=0.3)
    b = clada.window_attn(ctx, one.contiguous(), clada.KVCache(kc, vc), _ints([n, 30]), None, 20, 2, scale=0.3)
    assert torch.equal(a, b)


def test_a_row_past_2_31_values(clada, ctx):
    """A cache whose rows lie more than 2^31 values, and 2^32 bytes, from its start."""
    H, D, n = 2, 128, 300
    step = (2 ** 31 // n // 16 + 1) * 16
    base = [torch.zeros(step * n + H * D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    k, v = (torch.as_strided(x, (1, H, n, D), (0, D, step, 1)) for x in base)
    rng = np.random.default_rng(2)
    kc, vc = _draw(rng, "bf16", 1, H, n, D), _draw(rng, "bf16", 1, H, n, D)
    plan = clada.RopePlan(torch.zeros(4, dtype=torch.int64, device=DEV))                # turns of nothing: stored as they are
    clada.qk_rope(ctx, plan, None, kc.transpose(1, 2), vc.transpose(1, 2), torch.arange(n, dtype=torch.int32, device=DEV)[None], clada.KVCache(k, v))
    assert torch.equal(k, kc) and torch.equal(v, vc)
    for T in (1, 70):
        q = _draw(rng, "bf16", 1, T, 4, D)
        assert torch.equal(clada.window_attn(ctx, q, clada.KVCache(k, v), _ints([n])), clada.window_attn(ctx, q, clada.KVCache(kc, vc), _ints([n])))


@pytest.mark.parametrize("T", [1, 16, 200])
def test_same_bits_again_on_another_stream_and_in_a_graph(clada, ctx, T):
    rng = np.random.default_rng(T)
    B, Hq, H, D, n = 2, 8, 2, 128, 900
    q, kc, vc = _draw(rng, "bf16", B, T, Hq, D), _draw(rng, "bf16", B, H, n, D), _draw(rng, "bf16", B, H, n, D)
    cache, lens, out = clada.KVCache(kc, vc), _ints([n, n - 5]), torch.empty_like(q)
    first = clada.window_attn(ctx, q, cache, lens, window=700, sinks=4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = clada.window_attn(ctx, q, cache, lens, window=700, sinks=4)
        clada.graph_begin(ctx)
        clada.window_attn(ctx, q, cache, lens, window=700, sinks=4, out=out)
        g = clada.graph_end(ctx)
        for k in range(3):
            out.zero_()
            q.neg_()
            g.launch()
            s.synchronize()
            want = clada.window_attn(ctx, q, cache, lens, window=700, sinks=4)
            assert torch.equal(out, want) and torch.equal(want, first) == (k == 1)
    s.synchronize()
    assert torch.equal(first, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [900, 1024, 1025, 1160])
def test_joins_of_many_rows(clada, ctx, dtype, cap):
    """More than 1024 rows (four a compute unit) in eight splits and in nine and ten; sequences that leave splits, or everything, without keys."""
    _window_case(clada, ctx, dtype, 40, 8, 8, 48, [cap, 130, 0, 48], [48, 30, 0, 47], 0, 0, cap=cap, seed=cap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,H,B", [(80, 40, 2, 33), (256, 24, 3, 45)])
def test_shared_prefix_joins_of_many_rows(clada, ctx, dtype, D, Hq, H, B):
    test_shared_prefix(clada, ctx, dtype, D, Hq, H, B, 500)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,H,T,window,sinks,n_sink,ring", [(64, 2, 2, 64, 40, 1, 3, 110), (128, 4, 1, 32, 100, 4, 8, 131), (256, 1, 1, 40, 30, 2, 7, 75),
                                                               (96, 3, 1, 30, 60, 70, 75, 90)])
def test_rings_with_more_rows_of_their_own_than_sinks(clada, ctx, dtype, D, Hq, H, T, window, sinks, n_sink, ring):
    """Many rows, n_sink > sinks: a sequence of every length over a whole period of the ring, so that it wraps at every distance behind the sinks."""
    B, G = ring, Hq // H
    lens = [n_sink + 2 * ring + b for b in range(B)]
    rng = np.random.default_rng(ring)
    q = _draw(rng, dtype, B, T, Hq, D)
    kc, vc = (_draw(rng, dtype, B, H, n_sink + ring, D) for _ in range(2))
    out, lse = clada.window_attn(ctx, q, clada.KVCache(kc, vc, n_sink, ring), _ints(lens), None, window, sinks, want_lse=True)
    Q, K, V = to_np(q), to_np(kc), to_np(vc)
    r = dict(out=np.zeros(Q.shape), lse=np.zeros(Q.shape[:3]), mag=np.zeros(Q.shape), S=np.zeros(Q.shape[:3]), n=np.zeros(Q.shape[:3], int))
    for b in range(B):
        for t in range(T):
            pos = lens[b] - T + t
            rows = [ref.cache_row(p, n_sink, ring) for p in sorted({*range(pos - window + 1, pos + 1), *range(sinks)})]
            for h in range(Hq):
                r["out"][b, t, h], r["lse"][b, t, h], r["mag"][b, t, h], r["S"][b, t, h] = ref.attend(Q[b, t, h], K[b, h // G, rows], V[b, h // G, rows], D ** -0.5)
                r["n"][b, t, h] = len(rows)
    ref.check(to_np(out), to_np(lse), r, dtype, weights_bf16=True)


def _dense(q, k, v, scale, seen):
    """Rows q [..][r][D] over keys k, v [n][D] where seen [r][n], in 64 bits and laid out for ref.check."""
    k, v = k.double(), v.double()
    kt = k.t().contiguous()
    s = (scale * torch.matmul(q.double(), kt)).masked_fill(~seen, -float("inf"))
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None])
    S = abs(scale) * torch.matmul(q.double().abs(), kt.abs()).masked_fill(~seen, 0.0).amax(-1)
    r = {name: x.cpu().numpy() for name, x in dict(out=torch.matmul(p, v), lse=lse, mag=torch.matmul(p, v.abs()), S=S).items()}
    return dict(r, n=np.broadcast_to(seen.sum(-1).cpu().numpy(), lse.shape))


def _levels(kind, n, tile):
    """What the scores of n keys stand around, in powers of two."""
    x = np.zeros(n)
    if kind.startswith("rise"):                                 # from the middle of a tile on
        x[n // 3 + 5:] = float(kind[4:])
    elif kind == "stairs":
        x[n // 4:], x[n // 2:], x[3 * n // 4:] = 90, 220, 100
    elif kind == "pair":                                        # one key, then one of four times its weight in the tile behind it
        for a in range(3 * tile + 3, n - tile, n // 2):
            x[a], x[a + tile] = 126, 128
    return x


def _rising(rng, dtype, D, n, kind):
    """Keys and values [n][D] whose scores against a query that begins with a 4 stand around the levels of `kind`."""
    k, v = 0.3 * _draw(rng, dtype, n, D), _draw(rng, dtype, n, D)
    if kind == "lowest first":                                  # whole tiles of scores around -1e36: weights of exactly zero
        k[:n // 4, 0] = -1e36
    else:
        k[:, 0] = torch.from_numpy(_levels(kind, n, 64 if dtype == "bf16" and D <= 128 else 32) * np.log(2.0) * D ** 0.5 / 4.0).to(DEV)
    return k, v


RISES = ["rise70", "rise100", "rise127", "rise200", "stairs", "pair", "lowest first"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kind", RISES)
@pytest.mark.parametrize("B", [8, 16])                          # with 32 key heads: keys in two splits, in one
def test_many_rows_whose_scores_rise(clada, ctx, dtype, D, kind, B):
    """Scores that pass those of a row's first tile by any number of powers of two, in a tile that takes no maxima or in the one behind it."""
    rng = np.random.default_rng(D + B)
    H, T, n = 32, 20, 1024
    q = 0.3 * _draw(rng, dtype, B, T, H, D)
    q[..., 0] = 4.0
    k, v = _rising(rng, dtype, D, n, kind)
    cache = clada.KVCache(*(x.expand(B, H, n, D) for x in (k, v)))
    out, lse = clada.window_attn(ctx, q, cache, _ints([n] * B), want_lse=True)
    seen = torch.arange(n, device=DEV) <= torch.arange(n - T, n, device=DEV)[:, None]
    use = slice(n // 4 if kind == "lowest first" else 0, n)
    r = _dense(q.transpose(1, 2), k[use], v[use], D ** -0.5, seen[:, use])
    ref.check(to_np(out.transpose(1, 2)), to_np(lse.transpose(1, 2)), r, dtype, weights_bf16=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kind", RISES)
def test_a_shared_prefix_whose_scores_rise(clada, ctx, dtype, D, kind):
    """The same behind more than 16 rows a key head: eight splits of 512 rows whose sums stand at different powers of two."""
    rng = np.random.default_rng(D)
    B, H, n = 40, 32, 4096
    q = 0.3 * _draw(rng, dtype, B, H, D)
    q[..., 0] = 4.0
    k, v = _rising(rng, dtype, D, n, kind)
    cache = clada.KVCache(*(x[:1].expand(B, H, 1, D) for x in (k, v)))
    out, lse = clada.shared_prefix_attn(ctx, q, clada.KVCache(*(x.expand(1, H, n, D) for x in (k, v))), n, cache, _ints([0] * B), want_lse=True)
    use = slice(n // 4 if kind == "lowest first" else 0, n)
    r = _dense(q, k[use], v[use], D ** -0.5, torch.ones(1, n, dtype=torch.bool, device=DEV)[:, use])
    ref.check(to_np(out), to_np(lse), r, dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [0.0, 1e-38, -1e-39])
@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_scale_of_next_to_nothing(clada, ctx, dtype, T, scale, D):
    """Products of 1e37 and a scale that leaves nothing of them, or a few tenths: a float of 2^-149ths, 12 u of 1e-39, well within the d u of a score."""
    rng = np.random.default_rng(T)
    n = 200
    q, kc, vc = 2e18 * _draw(rng, dtype, 1, T, 2, D), 1e18 * _draw(rng, dtype, 1, 1, n, D), _draw(rng, dtype, 1, 1, n, D)
    out, lse = clada.window_attn(ctx, q, clada.KVCache(kc, vc), _ints([n]), scale=scale, want_lse=True)
    r = ref.window_attn(to_np(q), to_np(kc), to_np(vc), [n], [T], 0, 0, scale)
    ref.check(to_np(out), to_np(lse), r, dtype, weights_bf16=True)


@pytest.mark.parametrize("D,Hq,H,B", [(128, 8, 2, 3), (64, 4, 4, 1), (80, 5, 5, 17), (256, 8, 1, 5), (96, 6, 3, 40), (64, 40, 2, 2), (128, 16, 1, 64)])
@pytest.mark.parametrize("P", [1, 31, 500])
def test_a_shared_prefix_keeps_two_bf16_of_a_weight(clada, ctx, D, Hq, H, B, P):
    """The bound of weights of 16 bits, on few rows and on many."""
    rng = np.random.default_rng(D + B + P)
    q, lens = _draw(rng, "bf16", B, Hq, D), [int(v) for v in rng.integers(0, 41, B)]
    pk, pv = (_draw(rng, "bf16", 1, H, P, D) for _ in range(2))
    kc, vc = (_draw(rng, "bf16", B, H, 40, D) for _ in range(2))
    out, lse = clada.shared_prefix_attn(ctx, q, clada.KVCache(pk, pv), P, clada.KVCache(kc, vc), _ints(lens), want_lse=True)
    ref.check(to_np(out), to_np(lse), ref.shared_prefix_attn(to_np(q), to_np(pk)[0], to_np(pv)[0], P, to_np(kc), to_np(vc), lens, D ** -0.5), "bf16")


@pytest.mark.parametrize("D", [64, 96, 128, 200])
@pytest.mark.parametrize("T,Hq,H", [(2, 1, 1), (4, 8, 2), (16, 3, 3), (2, 8, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_up_to_sixteen_rows_keep_two_bf16_of_a_weight(clada, ctx, D, T, Hq, H, window, sinks):
    """Several queries, at most 16 rows a key head: the bound of weights of 16 bits."""
    rng = np.random.default_rng(D + T)
    lens, cap = [T, T + 100, T + 31, 330], 330
    q, kc, vc = _draw(rng, "bf16", 4, T, Hq, D), _draw(rng, "bf16", 4, H, cap, D), _draw(rng, "bf16", 4, H, cap, D)
    out, lse = clada.window_attn(ctx, q, clada.KVCache(kc, vc), _ints(lens), None, window, sinks, want_lse=True)
    ref.check(to_np(out), to_np(lse), ref.window_attn(to_np(q), to_np(kc), to_np(vc), lens, [T] * 4, window, sinks, D ** -0.5), "bf16")
