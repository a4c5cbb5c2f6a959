"""The paged cache's calls against the plain 64-bit implementations and their rounding bounds (paged_ref.py, attention_ref.py)."""
import numpy as np
import pytest
import torch

import attention_ref as ref
import paged_ref as paged
from gpu_util import DEV, to_dev, to_np

pytestmark = pytest.mark.gpu
TYPES = ["bf16", "f32", "mx4"]


@pytest.fixture(scope="module")
def clada():
    import paper_2502_19078_amd as pkg
    return pkg


@pytest.fixture(scope="module")
def ctx(clada):
    return clada.Context(0, clada.attn_workspace_bytes(64, 1024, 64, 256))


def _ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _np_dtype(kind):
    return "f32" if kind == "f32" else "bf16"


class Pool:
    """Pages of random values: the tensors of a PagedCache, and in 64 bits what they hold."""

    def __init__(self, clada, kind, P, H, page, D, table, seed=0, heads_last=False, pad=0):
        rng = np.random.default_rng(seed)
        self.kind, self.page = kind, page
        self.table = _ints(table)

        def tensor(width, dtype):                              # [P][H][page][width], maybe as [P][page][H][width], maybe with space behind
            shape = (P, page, H + pad, width) if heads_last else (P, H + pad, page, width)
            x = torch.zeros(shape, dtype=dtype, device=DEV)
            x = x.transpose(1, 2) if heads_last else x
            return x[:, :H]

        self.t = {}
        for n in "kv":
            x = rng.standard_normal((P, H, page, D))
            if kind == "mx4":
                x *= 2.0 ** rng.integers(-2, 3, (P, H, page, 1))
                code, byte = paged.quantise(x)
                self.t[n], self.t[n + "s"] = tensor(D // 2, torch.uint8), tensor(D // 32, torch.uint8)
                self.t[n].copy_(torch.from_numpy(paged.pack(code)))
                self.t[n + "s"].copy_(torch.from_numpy(byte.astype(np.uint8)))
            else:
                self.t[n], self.t[n + "s"] = tensor(D, torch.float32 if kind == "f32" else torch.bfloat16), None
                self.t[n].copy_(to_dev(x.astype(np.float32), kind))
        self.cache = clada.PagedCache(self.t["k"], self.t["v"], self.table, self.t["ks"], self.t["vs"])

    def held(self, n):
        """k or v [P][H][page][D] in 64 bits."""
        if self.kind == "mx4":
            return paged.values(paged.unpack(self.t[n].cpu().numpy()), self.t[n + "s"].cpu().numpy().astype(int))
        return to_np(self.t[n].contiguous())

    def spoil(self, n, at, value):
        """Rows at (pages, heads, rows) are not finite from here on (4 bits: NaN, whatever the value)."""
        if self.kind == "mx4":
            self.t[n + "s"][at] = 255
        else:
            self.t[n][at] = value


def _tables(rng, need, per, spare=2):
    """Tables that name `need` pages each, in no order, -1 behind; and the number of pages."""
    P = sum(need) + spare
    order = list(rng.permutation(P))
    rows = []
    for n in need:
        rows.append([order.pop() for _ in range(n)] + [-1] * (per - n))
    return rows, P


# ------------------------------------------------------------------------------------------------ append
def _near(got_code, got_byte, z, slack):
    """Whether codes and bytes are those of some value within slack of z [..., d]."""
    b, s = (x.reshape(*x.shape[:-1], -1, 32) for x in (np.abs(z), slack))
    low = np.vectorize(paged.block_byte, otypes=[int])(np.maximum(b - s, 0).max(-1))
    high = np.vectorize(paged.block_byte, otypes=[int])((b + s).max(-1))
    assert np.all((got_byte >= low) & (got_byte <= high))
    unit = 2.0 ** (got_byte - 127.0)[..., None]
    c = got_code.reshape(b.shape)
    assert np.all((c % 8 >= paged.nearest(np.maximum(b - s, 0) / unit)) & (c % 8 <= paged.nearest((b + s) / unit)))
    sign = np.signbit(z.reshape(b.shape))
    assert np.all(((c >= 8) == sign) | (b <= s))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("D,R,layout", [(128, 128, "half"), (128, 64, "half"), (128, 32, "half"), (128, 128, "pairs"), (64, 64, "half"), (96, 96, "half"), (96, 24, "half"),
                                        (256, 256, "half"), (32, 32, "half"), (160, 80, "pairs"), (192, 192, "half"), (64, 0, "half"), (224, 128, "half"), (80, 32, "pairs"),
                                        (72, 36, "half")])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("page,heads_last", [(16, False), (64, True)])
def test_append(clada, ctx, kind, D, R, layout, norm, page, heads_last):
    if kind == "mx4" and D % 32:
        pytest.skip("rows of 4 bits hold a multiple of 32 values")
    B, T, Hq, H = 3, 5, 6, 2
    pos = np.array([[0, 1, 2, 3, 4], [page - 2, page - 1, page, -1, 2 * page], [3 * page + 1, 5, 1 << 30, page * 2 - 1, 2147483647]])
    table = [[4, -1, -1, -1], [0, 6, 2, -1], [1, 3, 99, -7]]      # the third and fourth pages of the last sequence are not there
    pool = Pool(clada, kind, 7, H, page, D, table, seed=D + R, heads_last=heads_last, pad=1)
    before = {n: x.clone() for n, x in pool.t.items() if x is not None}
    dt = _np_dtype(kind)
    rng = np.random.default_rng(D)
    x = to_dev(rng.standard_normal((B, T, Hq + 2 * H, D)), dt)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
    w = [to_dev(1 + 0.2 * rng.standard_normal(D), dt) for _ in range(2)] if norm else [None, None]
    kw = dict(q_norm=w[0], k_norm=w[1], eps=1e-5, norm_offset=0.5) if norm else {}
    f, mag = ref.frequencies(R) if R else (np.zeros(0), 1.0)
    plan = clada.rope_plan(ctx, R, layout=clada.ROPE_HALF if layout == "half" else clada.ROPE_PAIRS) if R else \
        clada.RopePlan(torch.empty(0, dtype=torch.int64, device=DEV))
    out = clada.paged_rope(ctx, plan, q, k, v, _ints(pos), pool.cache, **kw)
    # the same arithmetic as the contiguous call's, bit for bit
    kc, vc = (torch.zeros((B, H, T, D), dtype=q.dtype, device=DEV) for _ in range(2))
    slots = np.where(pos < 0, -1, np.arange(T))
    want_q = clada.qk_rope(ctx, plan, q, k, v, _ints(pos), clada.KVCache(kc, vc), slots=_ints(slots), **kw)
    assert torch.equal(out, want_q)
    z = ref.rope(to_np(k), np.where(pos < 0, 0, pos), f, layout, mag, to_np(w[1]) if norm else None, 1e-5 if norm else None, 0.5)
    plain = np.abs(ref.rope(to_np(k), np.zeros_like(pos), f, layout, 1.0, to_np(w[1]) if norm else None, 1e-5 if norm else None, 0.5))
    if R:
        a, c = (slice(0, R // 2), slice(R // 2, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
        both = plain[..., a] + plain[..., c]
        plain[..., a], plain[..., c] = both, both
    slack = (D / 4 + 24) * 2.0 ** -24 * plain                   # test_gpu_rope's bound ahead of the last rounding
    for b in range(B):
        for t in range(T):
            p = pos[b, t]
            page_at = table[b][p // page] if 0 <= p < 4 * page else -1
            if not 0 <= page_at < 7:
                continue
            at = (page_at, slice(None), p % page)
            if kind == "mx4":
                _near(paged.unpack(pool.t["k"][at].cpu().numpy()), pool.t["ks"][at].cpu().numpy().astype(int), z[b, t], slack[b, t])
                code, byte = paged.quantise(to_np(v[b, t]))
                assert np.array_equal(pool.t["v"][at].cpu().numpy(), paged.pack(code)) and np.array_equal(pool.t["vs"][at].cpu().numpy(), byte)
            else:
                assert torch.equal(pool.t["k"][at], kc[b, :, t]) and torch.equal(pool.t["v"][at], vc[b, :, t])
            for n in before:
                before[n][at] = pool.t[n][at]
    for n in before:                                            # nothing else is touched
        assert torch.equal(before[n].view(torch.uint8) if kind == "mx4" else before[n], pool.t[n]), n


def test_append_keys_or_queries_alone(clada, ctx):
    pool = Pool(clada, "mx4", 3, 2, 16, 64, [[2, 0]], seed=1)
    q, k, v = (to_dev(np.random.default_rng(i).standard_normal((1, 20, 2, 64)), "bf16") for i in range(3))
    pos = _ints([list(range(20))])
    plan = clada.rope_plan(ctx, 64)
    before = {n: x.clone() for n, x in pool.t.items()}
    a = clada.paged_rope(ctx, plan, q, None, None, pos, pool.cache)
    assert all(torch.equal(before[n], pool.t[n]) for n in before)
    assert clada.paged_rope(ctx, plan, None, k, v, pos, pool.cache) is None
    alone = {n: x.clone() for n, x in pool.t.items()}
    for n in before:
        pool.t[n].copy_(before[n])
    out = torch.empty_like(q)
    assert clada.paged_rope(ctx, plan, q, k, v, pos, pool.cache, out=out) is out and torch.equal(out, a)
    assert all(torch.equal(alone[n], pool.t[n]) for n in before)


def test_append_of_what_is_not_finite(clada, ctx):
    """Only the block of such a value becomes NaN; zeros, and values below every exponent, are stored as such."""
    pool = Pool(clada, "mx4", 1, 1, 16, 128, [[0]], seed=1)
    v = np.random.default_rng(5).standard_normal((1, 6, 1, 128))
    v[0, 0, 0, 40], v[0, 1, 0, 0], v[0, 2, 0, 127] = np.nan, np.inf, -np.inf
    v[0, 3] = 0.0
    v[0, 4] = 2.0 ** -133
    v[0, 5, 0, :64] = 3.0e38
    vt = to_dev(v, "bf16")
    plan = clada.RopePlan(torch.empty(0, dtype=torch.int64, device=DEV))
    clada.paged_rope(ctx, plan, None, vt, vt, _ints([list(range(6))]), pool.cache)
    code, byte = paged.quantise(to_np(vt)[0, :, 0])
    for n in "kv":
        assert np.array_equal(pool.t[n + "s"][0, 0, :6].cpu().numpy(), byte)
        live = np.repeat(byte != 255, 16, -1)
        assert np.array_equal(pool.t[n][0, 0, :6].cpu().numpy()[live], paged.pack(code)[live])
    k, v2 = clada.paged_read(ctx, pool.cache, _ints([[0, 1, 2, 3, 4, 5]]))
    want = paged.values(code, byte)
    assert np.array_equal(to_np(v2)[0, :, 0], want, equal_nan=True) and np.array_equal(to_np(k)[0, :, 0], want, equal_nan=True)


# ------------------------------------------------------------------------------------------------ read
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("D", [32, 64, 80, 96, 128, 200, 256])
@pytest.mark.parametrize("page,heads_last", [(16, False), (128, True)])
def test_read(clada, ctx, kind, D, page, heads_last):
    if kind == "mx4" and D % 32:
        pytest.skip("rows of 4 bits hold a multiple of 32 values")
    H = 3
    table = [[4, 0, -1], [3, 12, 1]]
    pool = Pool(clada, kind, 6, H, page, D, table, seed=D, heads_last=heads_last)
    pos = [[0, page - 1, page, 2 * page, -1, 3 * page, 2147483647], [page, 2 * page + 3, 0, 0, 5, -9, 3 * page - 1]]
    want = {n: np.zeros((2, 7, H, D)) for n in "kv"}
    for b in range(2):
        for t, p in enumerate(pos[b]):
            if 0 <= p < 3 * page and 0 <= table[b][p // page] < 6:
                for n in "kv":
                    want[n][b, t] = pool.held(n)[table[b][p // page], :, p % page]
    k, v = clada.paged_read(ctx, pool.cache, _ints(pos))
    assert np.array_equal(to_np(k), want["k"]) and np.array_equal(to_np(v), want["v"])
    # one of them, into a cache's rows
    big = torch.full((2, H, 9, D), 7.0, dtype=k.dtype, device=DEV)
    into = big[:, :, 1:8].transpose(1, 2)
    assert clada.paged_read(ctx, pool.cache, _ints(pos), v_out=into)[0] is None
    assert np.array_equal(to_np(into), want["v"]) and torch.all(big[:, :, 0] == 7) and torch.all(big[:, :, 8] == 7)
    assert clada.paged_read(ctx, pool.cache, _ints(pos), k_out=into)[1] is None
    assert np.array_equal(to_np(into), want["k"])


# ------------------------------------------------------------------------------------------------ attention
def _case(clada, ctx, kind, D, Hq, H, T, lens, q_lens=None, page=16, seed=0, stale=float("nan"), heads_last=False, holes=(), max_len=0, scale=None,
          q_factor=1.0, **mods):
    """Random queries and pages; rows that no token has reached, pages of nobody and queries of padding hold `stale`."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    per = max(-(-max(lens) // page), 1) + 1
    table, P = _tables(rng, [-(-n // page) for n in lens], per)
    pool = Pool(clada, kind, P, H, page, D, table, seed=seed, heads_last=heads_last)
    held = np.zeros((P, page), bool)
    for b, n in enumerate(lens):
        for p in range(n):
            held[table[b][p // page], p % page] = True
    pages, rows = (torch.from_numpy(x).to(DEV) for x in np.nonzero(~held))
    for n in "kv":
        pool.spoil(n, (pages, slice(None), rows), stale)
    for b, j in holes:                                          # a page that is not there any more
        pool.table[b, j] = table[b][j] = [-1, P, 2147483647, -2147483648][(b + j) % 4]
    dt = _np_dtype(kind)
    q = to_dev(q_factor * rng.standard_normal((B, T, Hq, D)), dt)
    ql = q_lens if q_lens is not None else [T] * B
    for b in range(B):
        q[b, ql[b]:] = stale
    kw = dict(window=mods.get("window", 0), cap=mods.get("cap", 0.0))
    slopes = None
    if mods.get("bias"):
        slopes = np.float32(rng.uniform(0.0, mods["bias"], Hq))
        kw["slopes"] = torch.from_numpy(slopes).to(DEV)
    if "prefix" in mods:
        kw["prefix_lens"] = _ints(mods["prefix"])
    if "first" in mods:
        kw["first"] = _ints(mods["first"])
    scale = D ** -0.5 if scale is None else scale
    out, lse = clada.paged_attn(ctx, q, pool.cache, _ints(lens), None if q_lens is None else _ints(q_lens), max_len=max_len, scale=scale, want_lse=True, **kw)
    r = paged.paged_attn(to_np(q), pool.held("k"), pool.held("v"), table, page, lens, ql, scale, mods.get("window", 0), mods.get("cap", 0.0),
                         slopes, mods.get("prefix"), mods.get("first"), fp32=kind == "f32")
    ref.check(to_np(out), to_np(lse), r, dt, weights_bf16=T > 1)
    return out, lse


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("D", [8, 32, 64, 72, 80, 96, 128, 160, 192, 256])
@pytest.mark.parametrize("Hq,H", [(1, 1), (6, 2), (8, 1), (20, 1), (40, 1)])
def test_single_token(clada, ctx, kind, D, Hq, H):
    if kind == "mx4" and D % 32:
        pytest.skip("rows of 4 bits hold a multiple of 32 values")
    _case(clada, ctx, kind, D, Hq, H, 1, [1, 0, 37, 300, 129], page=16, seed=D + Hq)
    _case(clada, ctx, kind, D, Hq, H, 1, [300, 40, 33], page=64, seed=D + Hq + 1, heads_last=True, window=32, cap=3.0, bias=0.3)


MODS = [dict(), dict(window=1), dict(window=7), dict(window=64, cap=2.0), dict(cap=0.5), dict(cap=30.0, bias=0.5), dict(bias=1.5), dict(prefix=True), dict(first=True),
        dict(prefix=True, first=True, window=40, cap=5.0, bias=0.1)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("mods", MODS, ids=lambda m: "-".join(m) or "plain")
@pytest.mark.parametrize("T", [1, 2, 9, 33, 150])
def test_sight_and_scores(clada, ctx, kind, mods, T):
    """Lengths shorter than the queries (positions below zero), equal (a prompt), longer (a chunk), zero; ragged queries, none among them;
    documents that begin anywhere, also behind their query; prefixes of every length."""
    rng = np.random.default_rng(T)
    lens, q_lens = [T, T + 100, max(T - 1, 0), 0, T + 31], [T, T, T, T, max(T // 2, 0)]
    m = dict(mods)
    if "prefix" in m:
        m["prefix"] = [T // 2 + 1, T + 50, 1000, 5, 0]
    if "first" in m:
        m["first"] = [[int(rng.integers(-3, max(n, 1) + 2)) if t % 5 == 4 else max(0, (n - T + t) // 20 * 20) for t in range(T)] for n in lens]
    _case(clada, ctx, kind, 64, 4, 2, T, lens, q_lens, page=[16, 32][T % 2], seed=T + len(m), **m)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("D,Hq,H", [(128, 4, 1), (80, 3, 3), (256, 5, 1), (96, 7, 1), (64, 2, 1), (40, 2, 2), (200, 2, 1), (160, 2, 1), (32, 4, 2), (192, 2, 1)])
@pytest.mark.parametrize("T,extra", [(65, 0), (128, 1), (200, 77), (260, 0)])
def test_prompts(clada, ctx, kind, D, Hq, H, T, extra):
    if kind == "mx4" and D % 32:
        pytest.skip("rows of 4 bits hold a multiple of 32 values")
    _case(clada, ctx, kind, D, Hq, H, T, [T + extra, T // 2 + extra], [T, T // 2], page=16, seed=T + D)
    _case(clada, ctx, kind, D, Hq, H, T, [T + extra, T // 3], [T, T // 3], page=128, seed=T + D + 1, heads_last=True, window=50, cap=4.0, bias=0.2)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T", [1, 7, 40, 130])
@pytest.mark.parametrize("page", [16, 64])
def test_pages_that_are_not_there(clada, ctx, kind, T, page):
    """The first, the last and inner pages; all of a sequence's (its queries see nothing)."""
    n = T + 5 * page + 3
    last = (n - 1) // page
    _case(clada, ctx, kind, 64, 4, 2, T, [n, n, n - 1, page], page=page, seed=T, holes=[(0, 0), (0, 2), (1, 1), (1, 3), (2, last - 1), (3, 0)])
    _case(clada, ctx, kind, 64, 4, 2, T, [n, n], page=page, seed=T + 1, holes=[(0, last), (1, 0), (1, 1)], bias=0.2, cap=10.0, prefix=[n // 2, n])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T", [1, 20])
def test_long_sequences_are_split(clada, ctx, kind, T):
    """One sequence of 5000 keys among many workgroups, with and without a bound of the lengths; results are the same bits twice."""
    a = _case(clada, ctx, kind, 64, 4, 2, T, [5000, 1], page=32, seed=T, cap=20.0)
    b = _case(clada, ctx, kind, 64, 4, 2, T, [5000, 1], page=32, seed=T, cap=20.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    _case(clada, ctx, kind, 128, 4, 1, T, [1111, 40], page=32, seed=T, max_len=1200, bias=0.01)


@pytest.mark.parametrize("kind", TYPES)
def test_a_bound_of_the_lengths_cuts_them(clada, ctx, kind):
    pool = Pool(clada, kind, 4, 1, 16, 64, [[0, 1, 2, 3]], seed=3)
    q = to_dev(np.random.default_rng(3).standard_normal((1, 1, 2, 64)), _np_dtype(kind))
    whole = clada.paged_attn(ctx, q, pool.cache, _ints([40]))
    assert torch.equal(clada.paged_attn(ctx, q, pool.cache, _ints([64]), max_len=40), whole)
    assert torch.equal(clada.paged_attn(ctx, q, pool.cache, _ints([1000])), clada.paged_attn(ctx, q, pool.cache, _ints([64])))
    assert torch.all(clada.paged_attn(ctx, q, pool.cache, _ints([-5])) == 0)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T,window", [(1, 8), (5, 0), (40, 8), (150, 60)])
def test_what_is_masked_does_not_reach_the_output(clada, ctx, kind, bad, T, window):
    """A row of a page that is not finite reaches the queries that see it and no others."""
    rng = np.random.default_rng(7)
    D, Hq, H, page = 64, 4, 2, 16
    n = T + 20
    per = -(-n // page)
    pool = Pool(clada, kind, per, H, page, D, [list(range(per))[::-1]], seed=7)
    table = [list(range(per))[::-1]]
    q = to_dev(rng.standard_normal((1, T, Hq, D)), _np_dtype(kind))
    at = n - 1 - T // 3                                         # seen by the last third at most
    row = (table[0][at // page], slice(None), at % page)
    clean = pool.held("v").copy()
    if kind == "mx4":
        pool.t["vs"][row[0], :, row[2], 1] = 255                # values 32 to 63
    else:
        pool.t["v"][row[0], :, row[2], 5] = bad
    out, lse = clada.paged_attn(ctx, q, pool.cache, _ints([n]), window=window, want_lse=True)
    clean[row] = 0.0
    args = (table, page, [n], [T], D ** -0.5, window)
    r = paged.paged_attn(to_np(q), pool.held("k"), clean, *args)
    want = paged.paged_attn(to_np(q), pool.held("k"), pool.held("v"), *args)
    sees = np.array([at <= n - T + t and (window == 0 or at > n - T + t - window) for t in range(T)])
    got = to_np(out)
    assert np.array_equal(np.isnan(got), np.isnan(want["out"])) and np.array_equal(np.isposinf(got), np.isposinf(want["out"]))
    for t in np.nonzero(~sees)[0]:
        one = {k: v[:, t:t + 1] for k, v in r.items()}
        ref.check(got[:, t:t + 1], to_np(lse)[:, t:t + 1], one, _np_dtype(kind), weights_bf16=T > 1)
    # and a key that is not finite makes the scores of those queries so
    pool = Pool(clada, kind, per, H, page, D, table, seed=7)
    pool.spoil("k", (row[0], 0, row[2]), bad)
    out = to_np(clada.paged_attn(ctx, q, pool.cache, _ints([n]), window=window))
    assert np.all(np.isfinite(out[0, ~sees]))
    if bad != bad or kind == "mx4":
        assert np.all(np.isnan(out[0, sees][:, :Hq // H]))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 20])
def test_keys_of_the_lowest_value_and_scores_of_infinity(clada, ctx, kind, T):
    """A masked place may hold the type's lowest value; a query whose every score is -inf gives zeros; capped, infinities are numbers."""
    low = float(torch.finfo(torch.bfloat16 if kind == "bf16" else torch.float32).min)
    _case(clada, ctx, kind, 64, 4, 2, T, [T + 40, T + 3], page=16, seed=3, stale=low)
    pool = Pool(clada, kind, 4, 1, 16, 64, [[0, 1, 2, 3]], seed=3)
    q = torch.ones((1, T, 2, 64), dtype=pool.cache.dtype, device=DEV)
    pool.t["k"][:] = -float("inf")
    out, lse = clada.paged_attn(ctx, q, pool.cache, _ints([60]), want_lse=True)
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))
    out, lse = clada.paged_attn(ctx, q, pool.cache, _ints([60]), cap=5.0, want_lse=True)
    v = pool.held("v").transpose(1, 0, 2, 3).reshape(64, 64)
    for t in range(T):
        mean = v[:60 - T + t + 1].mean(0)
        assert np.allclose(to_np(out)[0, t], mean, atol=2.0 ** -7 if kind == "bf16" else 1e-5)
        assert np.allclose(to_np(lse)[0, t], -5.0 + np.log(60 - T + t + 1), atol=1e-5)


@pytest.mark.parametrize("kind", TYPES)
def test_scales_of_both_signs_and_zero(clada, ctx, kind):
    for T in (1, 40):
        for scale in (0.0, -0.2, 1e-38, 3.0):
            _case(clada, ctx, kind, 64, 4, 2, T, [T + 30, T], page=16, seed=5, scale=scale)
        _case(clada, ctx, kind, 64, 4, 2, T, [T + 30, T], page=16, seed=5, scale=-0.3, cap=2.0, bias=0.1)
        _case(clada, ctx, kind, 64, 4, 2, T, [T + 300, T], page=16, seed=5, scale=5.0, q_factor=8.0)      # scores of hundreds


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T", [1, 70])
def test_strided_queries_and_outputs(clada, ctx, kind, T):
    pool = Pool(clada, kind, 8, 2, 16, 64, [[0, 2, 4, 6, 1, 3, 5, 7]], seed=8, heads_last=True, pad=2)
    dt = _np_dtype(kind)
    big = to_dev(np.random.default_rng(1).standard_normal((1, T, 9, 64)), dt)
    q = big[:, :, 2:6]
    plain = clada.paged_attn(ctx, q.contiguous(), pool.cache, _ints([100]), cap=7.0)
    hold = torch.full((1, 6, T, 64), 3.0, dtype=q.dtype, device=DEV)
    out = hold[:, 1:5].transpose(1, 2)
    clada.paged_attn(ctx, q, pool.cache, _ints([100]), cap=7.0, out=out)
    assert torch.equal(out, plain) and torch.all(hold[:, 0] == 3) and torch.all(hold[:, 5] == 3)
    one = q[:, :, :1].expand(1, T, 4, 64)                       # a query that all heads share
    a = clada.paged_attn(ctx, one, pool.cache, _ints([100]), out=torch.empty((1, T, 4, 64), dtype=q.dtype, device=DEV))
    assert torch.equal(a, clada.paged_attn(ctx, one.contiguous(), pool.cache, _ints([100])))


def test_pages_far_into_a_pool(clada, ctx):
    """Offsets past 2^31 and 2^32 bytes."""
    P, H, page, D = 9000, 32, 64, 128                           # 4.7 GB each of k and v in bf16
    k = torch.zeros((P, H, page, D), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    near = [0, P // 2 + 100, P - 1]
    rng = np.random.default_rng(1)
    for p in near:
        k[p], v[p] = (to_dev(rng.standard_normal((H, page, D)), "bf16") for _ in range(2))
    cache = clada.PagedCache(k, v, _ints([near[::-1]]))
    small = clada.PagedCache(k[near].contiguous(), v[near].contiguous(), _ints([[2, 1, 0]]))
    q = to_dev(rng.standard_normal((1, 40, H, D)), "bf16")
    for n in (1, 40):
        assert torch.equal(clada.paged_attn(ctx, q[:, :n], cache, _ints([170])), clada.paged_attn(ctx, q[:, :n], small, _ints([170])))
    pos = _ints([[3, 70, 150]])
    assert all(torch.equal(a, b) for a, b in zip(clada.paged_read(ctx, cache, pos), clada.paged_read(ctx, small, pos)))
    plan = clada.rope_plan(ctx, D)
    x = to_dev(rng.standard_normal((1, 3, H, D)), "bf16")
    for c in (cache, small):
        clada.paged_rope(ctx, plan, None, x, x, pos, c)
    assert all(torch.equal(a, b) for a, b in zip(clada.paged_read(ctx, cache, pos), clada.paged_read(ctx, small, pos)))


@pytest.mark.parametrize("kind", TYPES)
def test_append_then_attend_as_a_server_does(clada, ctx, kind):
    """A prompt, a chunk and single tokens of two sequences, each appended and attended over, against one attention over all rows; then a
    sequence that shares the first one's full pages."""
    D, Hq, H, page = 64, 4, 2, 16
    rng = np.random.default_rng(11)
    dt = _np_dtype(kind)
    pool = Pool(clada, kind, 12, H, page, D, [[3, 1, 8, 0], [5, 2, 7, 9], [3, 1, 4, 6]], seed=2)
    plan = clada.rope_plan(ctx, D)
    n = [0, 0, 0]
    rows = to_dev(rng.standard_normal((3, 60, Hq + 2 * H, D)), dt)
    first = 0
    table = pool.table.tolist()
    for T, lens in ((30, [30, 21]), (9, [9, 9]), (1, [1, 1]), (1, [1, 1]), (1, [1, 0])):
        x = torch.zeros((2, T, Hq + 2 * H, D), dtype=rows.dtype, device=DEV)
        pos = np.full((2, T), -1)
        for b in range(2):
            x[b, :lens[b]] = rows[b, n[b]:n[b] + lens[b]]
            pos[b, :lens[b]] = np.arange(n[b], n[b] + lens[b])
            n[b] += lens[b]
        q = clada.paged_rope(ctx, plan, x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:], _ints(pos), pool.cache)
        out, lse = clada.paged_attn(ctx, q, pool.cache, _ints(n[:2]), _ints(lens), cap=8.0, want_lse=True)
        r = paged.paged_attn(to_np(q), pool.held("k"), pool.held("v"), table, page, n[:2], lens, D ** -0.5, cap=8.0, fp32=kind == "f32")
        ref.check(to_np(out), to_np(lse), r, dt, weights_bf16=T > 1)
    # the third sequence goes on from the first one's first 32 positions
    x = rows[2:3, :1]
    three = clada.PagedCache(pool.t["k"], pool.t["v"], pool.table[2:], pool.t["ks"], pool.t["vs"])
    q = clada.paged_rope(ctx, plan, x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:], _ints([[32]]), three)
    out, lse = clada.paged_attn(ctx, q, three, _ints([33]), want_lse=True)
    r = paged.paged_attn(to_np(q), pool.held("k"), pool.held("v"), table[2:], page, [33], [1], D ** -0.5)
    ref.check(to_np(out), to_np(lse), r, dt)
    # and its rows, read out of the pages, are a prefix for the contiguous call
    k, v = clada.paged_read(ctx, three, _ints([list(range(32))]))
    own = clada.paged_read(ctx, three, _ints([[32]]))
    kv = lambda a, b: clada.KVCache(a.transpose(1, 2).contiguous(), b.transpose(1, 2).contiguous())
    same, _ = clada.shared_prefix_attn(ctx, q[:, 0], kv(k, v), 32, kv(*own), _ints([1]), want_lse=True)
    ref.check(to_np(same)[:, None], None, r, dt)


@pytest.mark.parametrize("kind", TYPES)
def test_a_captured_step_replays(clada, kind):
    """Append and attend captured once; replays with new rows and lengths in the same buffers, eager work and synchronisations between."""
    D, Hq, H, page, B = 128, 8, 2, 16, 3
    ctx = clada.Context(0, clada.attn_workspace_bytes(B, 1, Hq, D))
    other = clada.Context(0, clada.attn_workspace_bytes(B, 1, Hq, D))
    rng = np.random.default_rng(4)
    pool, twin = (Pool(clada, kind, 40, H, page, D, np.arange(39).reshape(3, 13), seed=2) for _ in range(2))
    dt = _np_dtype(kind)
    rows = to_dev(rng.standard_normal((6, B, 1, Hq + 2 * H, D)), dt)
    plan = clada.rope_plan(ctx, D)
    x, pos, lens = rows[0].clone(), _ints([[100], [5], [190]]), _ints([101, 6, 191])
    out, q = torch.empty((B, 1, Hq, D), dtype=x.dtype, device=DEV), torch.empty((B, 1, Hq, D), dtype=x.dtype, device=DEV)

    def step(c, p, x, pos, lens, q, out):
        clada.paged_rope(c, plan, x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:], pos, p.cache, out=q)
        return clada.paged_attn(c, q, p.cache, lens, cap=20.0, out=out)

    step(ctx, pool, x, pos, lens, q, out)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        clada.graph_begin(ctx)
        step(ctx, pool, x, pos, lens, q, out)
        graph = clada.graph_end(ctx)
        for i in range(1, 6):
            x.copy_(rows[i])
            pos += 1
            lens += 1
            graph.launch()
            want = step(other, twin, rows[i], pos, lens, torch.empty_like(q), torch.empty_like(out))
            torch.cuda.synchronize()
            if i == 1:                                          # what the eager step ahead of the capture stored
                step(other, twin, rows[0], pos - 1, lens - 1, torch.empty_like(q), torch.empty_like(out))
                want = step(other, twin, rows[i], pos, lens, torch.empty_like(q), torch.empty_like(out))
            assert torch.equal(out, want), i
    torch.cuda.synchronize()


def test_two_streams_with_contexts_of_their_own(clada):
    D, Hq, H = 128, 8, 2
    pool = Pool(clada, "mx4", 40, H, 64, D, np.arange(40).reshape(1, 40), seed=2)
    q = to_dev(np.random.default_rng(1).standard_normal((1, 1, Hq, D)), "bf16")
    ctxs = [clada.Context(0, clada.attn_workspace_bytes(1, 1, Hq, D)) for _ in range(2)]
    lens = [_ints([2500]), _ints([1300])]
    want = [clada.paged_attn(c, q, pool.cache, n) for c, n in zip(ctxs, lens)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(clada.paged_attn(ctxs[i], q, pool.cache, lens[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for g, w in zip(got, want) for x in g)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cap,scale", [(50.0, None), (50.0, -0.1), (2.0, 0.3), (0.01, 0.2), (1e4, 1e-3), (1e-3, 30.0), (7.0, 0.0)])
def test_capped_prompts(clada, ctx, kind, cap, scale):
    """A cap alone, on tiles that every row sees: products far below it, around it and far above, scales of both signs and zero."""
    _case(clada, ctx, kind, 128, 4, 2, 200, [457, 200], page=64, seed=11, cap=cap, scale=scale)


@pytest.mark.parametrize("kind", TYPES)
def test_graphs_and_eager_calls_take_turns_with_one_workspace(clada, kind):
    """Two captured calls of different sizes, their keys split among workgroups, and an eager one on the same context: whatever the order, each finds the
    workspace as it needs it."""
    D, Hq, H, page = 64, 4, 2, 32
    shapes = [(1, 1, [4999]), (3, 2, [900, 2000, 31]), (2, 40, [700, 1300])]
    ctx = clada.Context(0, max(clada.attn_workspace_bytes(B, T, Hq, D) for B, T, _ in shapes))
    rng = np.random.default_rng(8)
    pool = Pool(clada, kind, 200, H, page, D, np.stack([rng.permutation(200)[:160] for _ in range(3)]), seed=5)
    qs = [to_dev(rng.standard_normal((B, T, Hq, D)), _np_dtype(kind)) for B, T, _ in shapes]
    lens, outs = [_ints(n) for _, _, n in shapes], [torch.zeros_like(q) for q in qs]

    def call(i, c, out):
        return clada.paged_attn(c, qs[i], pool.cache, lens[i], out=out)

    want = []
    for i, (B, T, _) in enumerate(shapes):
        alone = clada.Context(0, clada.attn_workspace_bytes(B, T, Hq, D))
        want.append(call(i, alone, torch.zeros_like(qs[i])))
        call(i, ctx, outs[i])
        torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graphs = []
        for i in (0, 1):
            clada.graph_begin(ctx)
            call(i, ctx, outs[i])
            graphs.append(clada.graph_end(ctx))
        for order in ((0, 1, 2), (1, 0, 2), (2, 0, 0, 1), (1, 2, 1, 0)):
            for out in outs:
                out.zero_()
            for i in order:
                graphs[i].launch() if i < 2 else call(2, ctx, outs[2])
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(outs, want)), order
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T", [1, 100])
def test_caps_at_the_ends_of_the_range(clada, ctx, kind, T):
    """A cap far above every score is none; one far below makes all weights equal."""
    D, H = 64, 2
    pool = Pool(clada, kind, 20, H, 16, D, np.arange(20).reshape(1, 20), seed=6)
    q = to_dev(np.random.default_rng(6).standard_normal((1, T, 4, D)), _np_dtype(kind))
    want, lse = clada.paged_attn(ctx, q, pool.cache, _ints([300]), want_lse=True)
    for cap in (3e38, 1e36, 1e33):
        got = clada.paged_attn(ctx, q, pool.cache, _ints([300]), cap=cap, want_lse=True)
        assert torch.equal(got[0], want) and torch.equal(got[1], lse), cap
    for cap in (1e-42, 1e-30):
        for scale in (None, -3.0):
            _case(clada, ctx, kind, D, 4, H, T, [300, 37 + T], page=16, seed=7, cap=cap, scale=scale)
