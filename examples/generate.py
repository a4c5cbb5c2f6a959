"""A decoder with random weights that generates for a batch of sequences behind one prompt, all heavy calls in the library.

    python examples/generate.py [--steps 32] [--batch 4] [--prompt 600] [--sparsity 0.45]

Layers alternate.  An even layer attends to everything: the prompt's keys and values are kept once for all sequences
(clada.shared_prefix_attn), each sequence has a cache for its own tokens.  An odd layer attends to a sliding window and the first tokens
(clada.window_attn) and keeps no more than those, in a ring.  clada.qk_rope norms and rotates queries and keys and fills the caches;
the FFN is CLADA's: dense over the prompt with its statistics (clada.prefix_stats, clada.threshold_calibrate), sparse for every
token after it (clada.signals_threshold, clada.sparse_ffn_decode).  Projections, norms and sampling are torch.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_19078_amd as clada  # noqa: E402


class Model:
    """L layers of width d, heads query heads on kv_heads key heads of head_dim values, window and sinks of the odd layers."""

    def __init__(self, L=4, d=512, d_ff=1376, V=1000, heads=8, kv_heads=2, head_dim=64, window=128, sinks=4, theta=10000.0, seed=0, dev="cuda:0"):
        g = torch.Generator().manual_seed(seed)
        mat = lambda *s: (torch.randn(*s, generator=g) * s[-1] ** -0.5).to(dev, torch.bfloat16)
        self.L, self.d, self.d_ff, self.V, self.heads, self.kv_heads, self.head_dim = L, d, d_ff, V, heads, kv_heads, head_dim
        self.window, self.sinks, self.theta, self.dev = window, sinks, theta, dev
        self.embed = mat(V, d) * d ** 0.5
        self.head = mat(V, d) * 2                            # logits of a few units
        self.qkv = [mat((heads + 2 * kv_heads) * head_dim, d) for _ in range(L)]
        self.out = [mat(d, heads * head_dim) for _ in range(L)]
        self.norm = [[(1 + 0.1 * torch.randn(head_dim, generator=g)).to(dev, torch.bfloat16) for _ in range(2)] for _ in range(L)]
        self.ffn = [clada.Layer(mat(d_ff, d), mat(d_ff, d), mat(d_ff, d)) for _ in range(L)]


def _rms(x):
    return (x.float() * torch.rsqrt(x.float().pow(2).mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Generator:
    def __init__(self, model: Model, prompt: torch.Tensor, batch: int, steps: int, sparsity: float):
        m = self.m = model
        P, rows = prompt.numel(), m.sinks + m.window
        need = max(clada.workspace_bytes(m.d, m.d_ff, batch, P, m.V), clada.attn_workspace_bytes(batch, 1, m.heads, m.head_dim),
                   clada.attn_workspace_bytes(1, P, m.heads, m.head_dim))
        self.ctx = clada.Context(0, need)
        self.plan = clada.rope_plan(self.ctx, m.head_dim, m.theta)
        self.P, self.batch = P, batch
        cache = lambda b, n, **kw: clada.KVCache(*(torch.zeros(b, m.kv_heads, n, m.head_dim, dtype=torch.bfloat16, device=m.dev) for _ in range(2)), **kw)
        self.prefix = [cache(1, P) for _ in range(m.L)]
        self.own = [cache(batch, steps) if l % 2 == 0 else cache(batch, rows, n_sink=m.sinks, ring=m.window) for l in range(m.L)]
        self.tau_base = torch.empty(m.L, device=m.dev)
        self.lam, self.gam = torch.full((m.L,), 0.8, device=m.dev), torch.full((m.L,), 0.12, device=m.dev)
        self.sparsity, self.n = sparsity, 0
        self.logits = self._prompt(prompt).expand(batch, m.V).contiguous()

    def _split(self, l, x, B, T):
        m = self.m
        h = (_rms(x) @ m.qkv[l].t()).view(B, T, m.heads + 2 * m.kv_heads, m.head_dim)
        return h[:, :, :m.heads], h[:, :, m.heads:m.heads + m.kv_heads], h[:, :, m.heads + m.kv_heads:]

    def _prompt(self, tokens):
        """The prompt through all layers: caches, and a base threshold for every layer; returns the last token's logits."""
        m, P = self.m, self.P
        x = m.embed[tokens]
        pos = torch.arange(P, dtype=torch.int32, device=m.dev)[None]
        length = torch.tensor([P], dtype=torch.int32, device=m.dev)
        for l in range(m.L):
            q, k, v = self._split(l, x, 1, P)
            q = clada.qk_rope(self.ctx, self.plan, q, k, v, pos, self.prefix[l], q_norm=m.norm[l][0], k_norm=m.norm[l][1])
            local = l % 2
            y = clada.window_attn(self.ctx, q, self.prefix[l], length, window=m.window if local else 0, sinks=m.sinks if local else 0)
            x = x + y.view(P, -1) @ m.out[l].t()
            s = clada.prefix_stats(self.ctx, m.ffn[l], _rms(x))
            clada.threshold_calibrate(self.ctx, s.abs_act_pool, self.sparsity, out=self.tau_base[l:l + 1])
            x = x + s.y
            if local:                                        # every sequence's ring begins with what the prompt leaves in the window
                p = torch.arange(P, device=m.dev)
                p = p[(p < m.sinks) | (p >= P - m.window)]
                row = torch.where(p < m.sinks, p, m.sinks + (p - m.sinks) % m.window)
                for to, src in ((self.own[l].k, self.prefix[l].k), (self.own[l].v, self.prefix[l].v)):
                    to[:, :, row] = src[:, :, p].expand(self.batch, -1, -1, -1)
        return (_rms(x[-1:]) @ m.head.t()).float()

    def step(self, tokens: torch.Tensor) -> torch.Tensor:
        """One token of every sequence; returns the logits behind it."""
        m, B, n = self.m, self.batch, self.n
        _, _, tau = clada.signals_threshold(self.ctx, self.logits, tokens, self.tau_base, self.lam, self.gam, math.log(m.V) / 2, math.log(m.V) / 2)
        x = m.embed[tokens.long()]
        ints = lambda v: torch.full((B,), v, dtype=torch.int32, device=m.dev)
        pos, own_row, own_len, length = ints(self.P + n), ints(n), ints(n + 1), ints(self.P + n + 1)
        for l in range(m.L):
            q, k, v = self._split(l, x, B, 1)
            q = clada.qk_rope(self.ctx, self.plan, q, k, v, pos, self.own[l], slots=None if l % 2 else own_row, q_norm=m.norm[l][0], k_norm=m.norm[l][1])
            if l % 2:
                y = clada.window_attn(self.ctx, q, self.own[l], length, window=m.window, sinks=m.sinks)
            else:
                y = clada.shared_prefix_attn(self.ctx, q[:, 0], self.prefix[l], self.P, self.own[l], own_len)
            x = x + y.reshape(B, -1) @ m.out[l].t()
            x = x + clada.sparse_ffn_decode(self.ctx, m.ffn[l], _rms(x), tau[l])
        self.n += 1
        self.logits = (_rms(x) @ m.head.t()).float()
        return self.logits


def main():
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=32)
    a.add_argument("--batch", type=int, default=4)
    a.add_argument("--prompt", type=int, default=600)
    a.add_argument("--sparsity", type=float, default=0.45)
    a = a.parse_args()
    model = Model()
    g = torch.Generator().manual_seed(1)
    prompt = torch.randint(model.V, (a.prompt,), generator=g).to(model.dev)
    gen = Generator(model, prompt, a.batch, a.steps, a.sparsity)
    gumbel = lambda: -torch.log(-torch.log(torch.rand(a.batch, model.V, generator=g).clamp(1e-9, 1 - 1e-7))).to(model.dev)
    out = []
    for _ in range(a.steps):
        tokens = (gen.logits + gumbel()).argmax(-1).to(torch.int32)
        out.append(tokens)
        gen.step(tokens)
    for b, row in enumerate(torch.stack(out, 1).tolist()):
        print(f"sequence {b}:", *row)


if __name__ == "__main__":
    main()
