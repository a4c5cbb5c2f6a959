"""The attention half of a decode step beside the library's FFN calls, timed call by call: position rotation into the key / value
cache, attention over the cache with a sliding window and sinks, attention of a batch over a prefix that all its sequences share.

Kinds of a case:

  rope     clada.qk_rope: norms of queries and keys for each head, rotary positions, keys and values stored into the cache
  window   clada.window_attn: T queries a sequence (1: a decode step) over its cache, causal, the last `window` positions (0: all)
           and the first `sinks`
  prefix   clada.shared_prefix_attn: one query a sequence over a prefix of P rows that the batch shares and its own rows

`own` False computes them with elementary torch operations in fp32, rounded once at the end; True with the library.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    bf = {"dtype": "bf16"}
    return [
        # one token of one sequence, 32 query and 8 key heads: launch latency only
        dict(name="rope_step_b1", kind="rope", B=1, T=1, Hq=32, Hkv=8, D=128, R=128, layout="half", scaling="none", norm=False,
             start=511, cap=1024, n_sink=0, ring=0, fused=True, **bf),
        # a prompt as long as the longest prefix of the configurations, norms for each head, frequencies scaled for long contexts
        dict(name="rope_prompt_t4096", kind="rope", B=1, T=4096, Hq=32, Hkv=8, D=128, R=128, layout="half", scaling="bands", norm=True,
             start=0, cap=4096, n_sink=0, ring=0, fused=True, **bf),
        # fp32 heads of 80 values of which 32 turn, neighbouring pairs, prompts of odd lengths padded to one
        dict(name="rope_ragged_f32", kind="rope", B=3, T=777, Hq=32, Hkv=32, D=80, R=32, layout="pairs", scaling="linear", norm=False,
             start=100, cap=1024, n_sink=0, ring=0, fused=False, dtype="f32"),
        # one token over a short prompt, eight query heads on one key head of 256 values: launch latency only
        dict(name="window_step_short", kind="window", B=1, T=1, Hq=8, Hkv=1, D=256, length=513, spread=0, cap=1024, window=0, sinks=0,
             n_sink=0, ring=0, **bf),
        # a decode step of eight sequences of different lengths with a window of 4096 and four sinks
        dict(name="window_step_b8", kind="window", B=8, T=1, Hq=32, Hkv=8, D=128, length=16384, spread=1801, cap=16384, window=4096,
             sinks=4, n_sink=0, ring=0, **bf),
        # one sequence of 128 Ki tokens, everything visible: the cache streams from HBM
        dict(name="window_step_128k", kind="window", B=1, T=1, Hq=32, Hkv=8, D=128, length=131071, spread=0, cap=131072, window=0,
             sinks=0, n_sink=0, ring=0, **bf),
        # chunks of 64 tokens into ring caches, small heads
        dict(name="window_chunk_ring", kind="window", B=4, T=64, Hq=16, Hkv=16, D=64, length=9001, spread=2500, cap=2116, window=2048,
             sinks=4, n_sink=4, ring=2112, **bf),
        # a prompt twice as long as its window: the largest case
        dict(name="window_prompt_t8192", kind="window", B=1, T=8192, Hq=32, Hkv=8, D=128, length=8192, spread=0, cap=8192, window=4096,
             sinks=4, n_sink=0, ring=0, **bf),
        # two fp32 prompts of odd lengths, heads of 80 values, a short window
        dict(name="window_prompt_f32", kind="window", B=2, T=1000, Hq=32, Hkv=32, D=80, length=1000, spread=263, cap=1000, window=256,
             sinks=4, n_sink=0, ring=0, dtype="f32"),
        # sixteen sequences behind one long instruction
        dict(name="prefix_b16", kind="prefix", B=16, P=8192, Hq=32, Hkv=8, D=128, length=512, spread=31, cap=512, **bf),
        # forty-eight short answers behind a shared document, every head with keys of its own
        dict(name="prefix_b48_heads32", kind="prefix", B=48, P=4095, Hq=32, Hkv=32, D=128, length=150, spread=3, cap=256, **bf),
        # a small fp32 batch, sizes odd
        dict(name="prefix_f32", kind="prefix", B=5, P=1001, Hq=12, Hkv=4, D=64, length=77, spread=15, cap=80, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    plain = 0                                                # values of the plain form's score matrix
    if c["kind"] == "window":
        plain = c["B"] * c["Hq"] * c["T"] * c["cap"]
    elif c["kind"] == "prefix":
        plain = c["B"] * c["Hq"] * (c["P"] + c["cap"])
    cache = c["B"] * c["Hkv"] * c["cap"] * c["D"]
    return max(w["bytes"] / 5.4e8, w["flops"] / 4.1e11, plain / 2.1e9, cache / 1.35e8)       # about 1 for the listed case that has most of each


_LARGEST = None


def draw(rng):
    """One more case of the same ranges: lengths, batches, head layouts and windows away from the listed ones."""
    global _LARGEST
    if _LARGEST is None:
        _LARGEST = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["rope", "window", "window", "window", "prefix"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        D = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
        Hkv = rng.choice([1, 2, 4, 5, 8, 8, 16, 32])
        G = rng.choice([1, 2, 3, 4, 4, 7, 8])
        c = dict(kind=kind, Hq=Hkv * G, Hkv=Hkv, D=D, dtype=dtype)
        if c["Hq"] > 64:
            continue
        if kind == "rope":
            T = 1 if rng.random() < 0.4 else _log_int(rng, 2, 8192)
            B = _log_int(rng, 1, 64) if T == 1 else _log_int(rng, 1, 8)
            start = 0 if rng.random() < 0.4 else _log_int(rng, 1, 100000)
            n_sink, ring = (4, _log_int(rng, T, 2 * T + 1000)) if rng.random() < 0.3 else (0, 0)
            if not ring and start > 4096:                    # a plain cache holds every position
                start = _log_int(rng, 1, 4096)
            cap = n_sink + ring if ring else start + T + rng.randint(0, 64)
            c.update(B=B, T=T, R=rng.choice([D, D, D // 2 // 2 * 2, 16, 32, 24]), layout=rng.choice(["half", "half", "pairs"]),
                     scaling=rng.choice(["none", "linear", "base", "bands", "ramp"]), norm=rng.random() < 0.5, start=start, cap=cap,
                     n_sink=n_sink, ring=ring, fused=rng.random() < 0.5)
        elif kind == "window":
            form = rng.choice(["step", "step", "chunk", "prompt"])
            T = {"step": 1, "chunk": _log_int(rng, 2, 256), "prompt": _log_int(rng, 16, 8192)}[form]
            B = _log_int(rng, 1, 64 if form == "step" else 8)
            length = T if form == "prompt" else T + _log_int(rng, 1, 131072 if form == "step" else 16384)
            window = 0 if rng.random() < 0.35 else _log_int(rng, 16, 8192)
            sinks = rng.choice([0, 1, 4, 16]) if window else 0
            n_sink, ring = (sinks, window + T + rng.randint(0, 100)) if window and rng.random() < 0.3 else (0, 0)
            spread = rng.randint(0, max(0, length - 1) // B) if B > 1 else 0
            cap = n_sink + ring if ring else length + rng.randint(0, 64)
            c.update(B=B, T=T, length=length, spread=spread, cap=cap, window=window, sinks=sinks, n_sink=n_sink, ring=ring)
        else:
            length = _log_int(rng, 1, 1024)
            B = _log_int(rng, 1, 64)
            c.update(B=B, P=_log_int(rng, 16, 32768), length=length, spread=rng.randint(0, length // B), cap=length + rng.randint(0, 64))
        if _cost(c) <= _LARGEST:
            return c


# ------------------------------------------------------------------------------------------------ sizes that a case implies
def _lens(c):
    """Tokens of every sequence: the first has `length`, each further one `spread` fewer."""
    return [max(0, c["length"] - c["spread"] * b) for b in range(c["B"])]


def _q_lens(c):
    """Queries of every sequence: T, or as many as it has tokens."""
    return [min(c["T"], n) for n in _lens(c)]


def _rope_tokens(c):
    """Tokens of every sequence of a prompt: each a little shorter than the one before, padded to T."""
    return [max(1, c["T"] - b * (c["T"] // 7)) for b in range(c["B"])]


def _visible(n, queries, window, sinks):
    """(pairs, rows seen by any) of the last `queries` of n causal tokens."""
    if not queries:
        return 0, 0
    first = n - queries
    recent = [min(pos + 1, window) if window else pos + 1 for pos in range(first, n)]
    pairs = sum(r + min(sinks, pos + 1 - r) for pos, r in zip(range(first, n), recent))
    oldest = max(0, first - window + 1) if window else 0
    return pairs, n - oldest + min(sinks, oldest)


def work(c):
    es = 4 if c["dtype"] == "f32" else 2
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "rope":
        n = sum(_rope_tokens(c))
        values = n * (Hq + Hkv) * D
        # one read and one write of the queries, keys and values; squares, scaling and rotation; two functions an angle
        return {"bytes": 2 * es * n * (Hq + 2 * Hkv) * D + 4 * n + 4 * c["R"], "flops": (4 if c["norm"] else 0) * values + 3 * n * (Hq + Hkv) * c["R"]}
    if c["kind"] == "window":
        pairs = rows = 0
        for n, t in zip(_lens(c), _q_lens(c)):
            p, r = _visible(n, t, c["window"], c["sinks"])
            pairs, rows = pairs + p, rows + r
        io = c["B"] * c["T"] * Hq
        return {"bytes": es * (2 * io * D + 2 * rows * Hkv * D) + 4 * io, "flops": 4 * D * Hq * pairs}
    rows = sum(_lens(c))
    io = c["B"] * Hq
    return {"bytes": es * (2 * io * D + 2 * (c["P"] + rows) * Hkv * D) + 4 * io, "flops": 4 * D * Hq * (c["B"] * c["P"] + rows)}


# ------------------------------------------------------------------------------------------------ inputs
def _frequencies(R, scaling):
    """(angle a position of every pair, factor of the cosines and sines): theta^(-2i/R), scaled for contexts eight times as long."""
    theta, factor, original = 10000.0, 8.0, 4096.0
    if scaling == "base" and R > 2:
        theta *= factor ** (R / (R - 2))
    f = [theta ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    elif scaling == "bands":                                 # short waves stay, long ones are stretched, a blend between
        low, high = 1.0, 4.0
        blend = [min(1.0, max(0.0, (original * x / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [(1 - s) * x / factor + s * x for x, s in zip(f, blend)]
    elif scaling == "ramp":                                  # blended by the pair's index between two wave counts
        at = lambda turns: R * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), R - 1)
        keep = [1 - min(1.0, max(0.0, (i - low) / max(high - low, 0.001))) for i in range(R // 2)]
        f = [x / factor * (1 - s) + x * s for x, s in zip(f, keep)]
    return f, (0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0)


def _turns(f):
    """Angles as 2^64ths of a turn, which a product with a position wraps exactly; the bits of an unsigned number in an int64."""
    v = [round(x / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for x in f]
    return torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in v], dtype=torch.int64)


def _device():
    return "cuda:0" if torch.cuda.is_available() else "cpu"


def _inputs(c, seed):
    """Every tensor of a case from its seed.  Queries and keys share a direction as trained ones do, the first keys most of all, so
    that the weights are neither flat nor one; rows of a cache that no token has reached hold what another request left there."""
    dev, dt = _device(), _DT[c["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device=dev, dtype=torch.float32)
    B, Hq, Hkv, D, G = c["B"], c["Hq"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    if c["kind"] == "rope":
        T = c["T"]
        f, magnitude = _frequencies(c["R"], c["scaling"])
        if c["fused"]:                                       # one projection's output: queries, keys and values side by side
            x = normal(B, T, Hq + 2 * Hkv, D).to(dt)
            q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
        else:
            q, k, v = (normal(B, T, h, D).to(dt) for h in (Hq, Hkv, Hkv))
        start, n = c["start"], _rope_tokens(c)
        t = torch.arange(T, device=dev, dtype=torch.int32)
        pos = torch.stack([torch.where(t < n[b], t + start, -1) for b in range(B)]).contiguous()
        w = [(1 + 0.1 * normal(D)).to(dt) for _ in range(2)] if c["norm"] else [None, None]
        return dict(q=q, k=k, v=v, pos=pos, qw=w[0], kw=w[1], turns=_turns(f).to(dev), f=f, magnitude=magnitude,
                    kc=normal(B, Hkv, c["cap"], D).to(dt), vc=normal(B, Hkv, c["cap"], D).to(dt))
    common = normal(Hkv, D)
    keys = lambda *s: 0.9 * normal(*s) + 0.4 * common[:, None]
    if c["kind"] == "window":
        q = 1.3 * normal(B, c["T"], Hkv, G, D) + 0.4 * common[:, None]
        k, v = keys(B, Hkv, c["cap"], D), normal(B, Hkv, c["cap"], D) + 0.1 * normal(Hkv, 1, D)
        k[:, :, :c["sinks"]] += 0.5 * common[:, None]
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
        return dict(q=q.reshape(B, c["T"], Hq, D).to(dt), kc=k.to(dt), vc=v.to(dt), lens=i32(_lens(c)), q_lens=i32(_q_lens(c)))
    q = 1.3 * normal(B, Hkv, G, D) + 0.4 * common[:, None]
    k, v, pk, pv = keys(B, Hkv, c["cap"], D), normal(B, Hkv, c["cap"], D), keys(1, Hkv, c["P"], D), normal(1, Hkv, c["P"], D)
    return dict(q=q.reshape(B, Hq, D).to(dt), kc=k.to(dt), vc=v.to(dt), pk=pk.to(dt), pv=pv.to(dt),
                lens=torch.tensor(_lens(c), dtype=torch.int32, device=dev))


def prepare(case, seed):
    return dict(_inputs(case, seed), case=dict(case))


# ------------------------------------------------------------------------------------------------ plain forms
def _slot(c, pos):
    """Cache row of a position: itself, or in a ring behind the first n_sink rows."""
    if not c["ring"]:
        return pos
    return torch.where(pos < c["n_sink"], pos, c["n_sink"] + (pos - c["n_sink"]) % c["ring"])


def _plain_rope(s):
    c = s["case"]
    D, R = c["D"], c["R"]
    pos = s["pos"].long()
    turns = ((pos.clamp(min=0)[..., None] * s["turns"]) >> 32).float() * (2 * math.pi * 2.0 ** -32)
    cos, sin = (s["magnitude"] * turns.cos())[:, :, None], (s["magnitude"] * turns.sin())[:, :, None]

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        a, b = (x[..., :R // 2], x[..., R // 2:R]) if c["layout"] == "half" else (x[..., 0:R:2], x[..., 1:R:2])
        a, b = a * cos - b * sin, b * cos + a * sin
        y = torch.cat([a, b], -1) if c["layout"] == "half" else torch.stack([a, b], -1).flatten(-2)
        return torch.cat([y, x[..., R:]], -1)

    live = pos >= 0
    q = torch.where(live[:, :, None, None], turned(s["q"], s["qw"]), 0.0).to(s["q"].dtype)
    k = turned(s["k"], s["kw"]).to(s["k"].dtype)
    b, t = torch.nonzero(live, as_tuple=True)
    row = _slot(c, pos[b, t])
    s["kc"][b, :, row] = k[b, t]
    s["vc"][b, :, row] = s["v"][b, t]
    return {"q": q, "k_cache": s["kc"], "v_cache": s["vc"]}


def _softmax(x, seen):
    """(weights, log of their sum) over the last axis where `seen`; a row that sees nothing has zero weights and -inf."""
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total), (m + torch.log(total)).squeeze(-1)


def _plain_window(s):
    c = s["case"]
    B, T, Hq, Hkv, D, cap = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"], c["cap"]
    G, dev = Hq // Hkv, s["q"].device
    n, t = s["lens"].long()[:, None], torch.arange(T, device=dev)
    pos = n - s["q_lens"].long()[:, None] + t                # [B][T]
    pos = torch.where(t < s["q_lens"].long()[:, None], pos, -1)
    slot = torch.arange(cap, device=dev)
    held = slot[None] + 0 * n                                # the position that a row of the cache holds, [B][cap]
    if c["ring"]:
        last = n - 1 - c["n_sink"]
        held = torch.where(slot < c["n_sink"], held, n - 1 - (last - (slot - c["n_sink"])) % c["ring"])
        held = torch.where((slot >= c["n_sink"]) & (held < c["n_sink"]), n, held)
    held, at = held[:, None], pos[:, :, None]
    seen = held <= at
    if c["window"]:
        seen = seen & ((held > at - c["window"]) | (held < c["sinks"]))
    q = s["q"].float().view(B, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T, D)
    x = torch.matmul(q, s["kc"].float().transpose(-1, -2)).mul_(D ** -0.5).view(B, Hkv, G, T, cap)
    p, lse = _softmax(x, seen[:, None, None])
    v = torch.where((slot < n)[:, None, :, None], s["vc"].float(), 0.0)
    o = torch.matmul(p.view(B, Hkv, G * T, cap), v).view(B, Hkv, G, T, D).permute(0, 3, 1, 2, 4)
    return {"out": o.reshape(B, T, Hq, D).to(s["q"].dtype), "lse": lse.permute(0, 3, 1, 2).reshape(B, T, Hq).contiguous()}


def _plain_prefix(s):
    c = s["case"]
    B, P, Hq, Hkv, D, cap = c["B"], c["P"], c["Hq"], c["Hkv"], c["D"], c["cap"]
    G = Hq // Hkv
    q = s["q"].float().view(B, Hkv, G, D) * D ** -0.5
    shared = torch.matmul(q.transpose(0, 1).reshape(Hkv, B * G, D), s["pk"][0].float().transpose(-1, -2))
    mine = torch.matmul(q, s["kc"].float().transpose(-1, -2))
    x = torch.cat([shared.view(Hkv, B, G, P).transpose(0, 1), mine], -1)
    seen = torch.arange(P + cap, device=q.device) < P + s["lens"].long()[:, None]
    p, lse = _softmax(x, seen[:, None, None])
    o = torch.matmul(p[..., :P].transpose(0, 1).reshape(Hkv, B * G, P), s["pv"][0].float()).view(Hkv, B, G, D).transpose(0, 1)
    o = o + torch.matmul(p[..., P:], s["vc"].float())
    return {"out": o.reshape(B, Hq, D).to(s["q"].dtype), "lse": lse.reshape(B, Hq)}


# ------------------------------------------------------------------------------------------------ the library's calls
_CONTEXT = []


def _context(clada):
    """The handle that a program keeps: one context, its workspace as large as these calls make use of."""
    if not _CONTEXT:
        _CONTEXT.append(clada.Context(0, clada.attn_workspace_bytes(64, 8192, 64, 256)))
    return _CONTEXT[0]


def _own(s):
    import paper_2502_19078_amd as clada

    c, ctx = s["case"], _context(clada)
    if c["kind"] == "rope":
        plan = clada.RopePlan(s["turns"], clada.ROPE_HALF if c["layout"] == "half" else clada.ROPE_PAIRS, s["magnitude"])
        cache = clada.KVCache(s["kc"], s["vc"], n_sink=c["n_sink"], ring=c["ring"])
        q = clada.qk_rope(ctx, plan, s["q"], s["k"], s["v"], s["pos"], cache, q_norm=s["qw"], k_norm=s["kw"], eps=1e-6)
        return {"q": q, "k_cache": s["kc"], "v_cache": s["vc"]}
    if c["kind"] == "window":
        cache = clada.KVCache(s["kc"], s["vc"], n_sink=c["n_sink"], ring=c["ring"])
        out, lse = clada.window_attn(ctx, s["q"], cache, s["lens"], q_lens=s["q_lens"], window=c["window"], sinks=c["sinks"], want_lse=True)
        return {"out": out, "lse": lse}
    out, lse = clada.shared_prefix_attn(ctx, s["q"], clada.KVCache(s["pk"], s["pv"]), c["P"], clada.KVCache(s["kc"], s["vc"]), s["lens"],
                                        want_lse=True)
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "window": _plain_window, "prefix": _plain_prefix}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_rows(q, k, v, seen, scale):
    """Attention of rows q [n][D] over k, v [m][D] where seen [n][m]."""
    x = (q @ k.t().contiguous()) * scale
    x.masked_fill_(~seen, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[:, None])
    p[lse == -math.inf] = 0.0
    return p @ v, lse


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    G, d64 = Hq // Hkv, torch.float64
    if c["kind"] == "rope":
        R, dev = c["R"], s["q"].device
        f = torch.tensor(s["f"], dtype=d64, device=dev)
        q, k, v = (s[n].to(d64) for n in ("q", "k", "v"))
        kc, vc = s["kc"].to(d64), s["vc"].to(d64)
        if c["norm"]:
            q = q / torch.sqrt(q.pow(2).mean(-1, keepdim=True) + 1e-6) * s["qw"].to(d64)
            k = k / torch.sqrt(k.pow(2).mean(-1, keepdim=True) + 1e-6) * s["kw"].to(d64)
        i = torch.arange(R // 2, device=dev)
        first, second = (i, i + R // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        angle = s["pos"].to(d64)[..., None] * f
        turn = s["magnitude"] * torch.polar(torch.ones_like(angle), angle)[:, :, None]
        for x in (q, k):
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
        q[s["pos"] < 0] = 0.0
        pos = s["pos"].tolist()
        for b, row in enumerate(pos):
            live = [t for t, p in enumerate(row) if p >= 0]
            to = [p if not c["ring"] or p < c["n_sink"] else c["n_sink"] + (p - c["n_sink"]) % c["ring"] for p in row if p >= 0]
            kc[b, :, to] = k[b, live].transpose(0, 1)
            vc[b, :, to] = v[b, live].transpose(0, 1)
        return {"q": q, "k_cache": kc, "v_cache": vc}
    if c["kind"] == "window":
        if c["B"] * Hq * c["T"] * c["length"] > 3e9:
            return None
        out = torch.zeros(s["q"].shape, dtype=d64, device=s["q"].device)
        lse = torch.full(s["q"].shape[:3], -math.inf, dtype=d64, device=s["q"].device)
        for b, (n, t) in enumerate(zip(_lens(c), _q_lens(c))):
            if not t:
                continue
            p = torch.arange(n, device=out.device)
            at = p[n - t:, None]
            seen = p <= at
            oldest = 0
            if c["window"]:
                seen &= (p > at - c["window"]) | (p < c["sinks"])
                oldest = max(0, n - t - c["window"] + 1)
            ring = c["ring"] or max(n, 1)
            base = c["n_sink"] if c["ring"] else 0
            row = torch.where(p < base, p, base + (p - base) % ring)
            use = (p >= oldest) | (p < c["sinks"])           # rows of a ring that positions before these held are gone
            row, seen = row[use], seen[:, use].repeat(G, 1)
            for h in range(Hkv):
                q = s["q"][b, :t, h * G:(h + 1) * G].to(d64).transpose(0, 1).reshape(G * t, D)
                o, l = _exact_rows(q, s["kc"][b, h, row].to(d64), s["vc"][b, h, row].to(d64), seen, 1 / math.sqrt(D))
                out[b, :t, h * G:(h + 1) * G] = o.view(G, t, D).transpose(0, 1)
                lse[b, :t, h * G:(h + 1) * G] = l.view(G, t).t()
        return {"out": out, "lse": lse}
    out = torch.zeros(s["q"].shape, dtype=d64, device=s["q"].device)
    lse = torch.zeros(s["q"].shape[:2], dtype=d64, device=s["q"].device)
    for h in range(Hkv):
        pk, pv = s["pk"][0, h].to(d64), s["pv"][0, h].to(d64)
        for b, n in enumerate(_lens(c)):
            k, v = torch.cat([pk, s["kc"][b, h, :n].to(d64)]), torch.cat([pv, s["vc"][b, h, :n].to(d64)])
            seen = torch.ones(G, c["P"] + n, dtype=torch.bool, device=out.device)
            out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = _exact_rows(s["q"][b, h * G:(h + 1) * G].to(d64), k, v, seen, 1 / math.sqrt(D))
    return {"out": out, "lse": lse}
