"""CPU-only checks of the cache and attention calls: what they refuse, with which status, before any GPU is touched, and what the binding
refuses by itself; clada_rope_turns, which runs on the host, against 64-bit frequencies."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import attention_ref as ref

OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, VALUE = 0, 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def b():
    import paper_2502_19078_amd as pkg
    if not os.path.exists(pkg.lib_path()):
        from paper_2502_19078_amd import build
        build.build()
    pkg.load_library()
    import paper_2502_19078_amd.binding as binding
    return binding


class Calls:
    """The three calls on a context without a device, each argument replaceable by name."""

    def __init__(self, b):
        self.b, self.lib = b, b.load_library()
        self.h = C.c_void_p()
        assert self.lib.clada_create(C.byref(self.h), 0, 0) == OK
        self.buf = (C.c_char * 8192)()
        self.p = (C.addressof(self.buf) + 255) // 256 * 256
        self.heads = dict(data=self.p, stride_b=4096, stride_t=1024, stride_h=128)
        self.kv = dict(k=self.p, v=self.p, stride_b=65536, stride_h=8192, stride_n=128, batch=2, heads=2, d=128, capacity=64, dtype=b.BF16, n_sink=0, ring=0)
        self.rope = dict(turns=self.p, rotary_dim=64, layout=0, magnitude=1.0)

    def _s(self, cls, base, change):
        return None if change is None else C.byref(cls(**{**base, **change}))

    def qk_rope(self, q={}, k={}, v={}, out={}, cache={}, rope={}, norm=None, B=2, T=3, Hq=4, pos=True, slots=None):
        b, H = self.b, lambda x: self._s(b._CHeads, self.heads, x)
        n = None if norm is None else C.byref(b._CHeadNorm(**{**dict(q_weight=self.p, k_weight=self.p, eps=1e-6, offset=0.0), **norm}))
        return self.lib.clada_qk_rope(self.h, self._s(b._CRope, self.rope, rope), n, B, T, Hq, H(q), H(k), H(v), self.p if pos is True else pos, slots, H(out),
                                      self._s(b._CKvCache, self.kv, cache), None)

    def window(self, q={}, out={}, cache={}, lens=True, q_lens=None, B=2, T=1, Hq=4, window=0, sinks=0, scale=1.0, lse=None):
        b = self.b
        return self.lib.clada_window_attn(self.h, self._s(b._CHeads, self.heads, q), self._s(b._CKvCache, self.kv, cache), self.p if lens is True else lens, q_lens, B, T,
                                          Hq, window, sinks, scale, self._s(b._CHeads, self.heads, out), lse, None)

    def prefix(self, q={}, out={}, prefix={}, cache={}, lens=True, n=64, B=2, Hq=4, scale=1.0, lse=None):
        b = self.b
        return self.lib.clada_shared_prefix_attn(self.h, self._s(b._CHeads, self.heads, q), self._s(b._CKvCache, self.kv, prefix), n,
                                                 self._s(b._CKvCache, self.kv, cache), self.p if lens is True else lens, B, Hq, scale,
                                                 self._s(b._CHeads, self.heads, out), lse, None)


def test_refusals(b):
    c = Calls(b)
    p = c.p
    # accepted up to the missing device
    assert c.qk_rope() == c.qk_rope(norm={}) == c.qk_rope(q=None, out=None) == c.qk_rope(k=None, v=None) == WORKSPACE
    assert c.qk_rope(rope=dict(turns=None, rotary_dim=0)) == c.qk_rope(slots=p) == WORKSPACE
    assert c.window() == c.window(T=9, q_lens=p, window=5, sinks=2, lse=p) == c.window(cache=dict(n_sink=4, ring=60), window=60, sinks=4) == WORKSPACE
    assert c.prefix() == c.prefix(lse=p, prefix=dict(batch=1, capacity=70)) == WORKSPACE
    # no context, missing pointers
    assert c.lib.clada_window_attn(None, None, None, None, None, 1, 1, 1, 0, 0, 1.0, None, None, None) == NULL
    assert c.lib.clada_rope_turns(None, 2, None, None, None) == NULL
    for bad in (dict(q=None, k=None, v=None, out=None), dict(out=None), dict(v=None), dict(k=None), dict(pos=None), dict(cache=None), dict(rope=None),
                dict(q=dict(data=None)), dict(cache=dict(k=None)), dict(rope=dict(turns=None))):
        assert c.qk_rope(**bad) == NULL, bad
    for bad in (dict(q=None), dict(out=None), dict(cache=None), dict(lens=None), dict(cache=dict(v=None)), dict(out=dict(data=None))):
        assert c.window(**bad) == NULL, bad
    for bad in (dict(q=None), dict(prefix=None), dict(cache=None), dict(lens=None), dict(prefix=dict(k=None))):
        assert c.prefix(**bad) == NULL, bad
    # sizes
    kv = [dict(d=4), dict(d=100), dict(d=264), dict(batch=0), dict(heads=0), dict(heads=1025), dict(capacity=0), dict(capacity=(1 << 30) + 1), dict(n_sink=-1), dict(ring=-1),
          dict(n_sink=4, ring=61), dict(stride_n=-128)]
    for bad in kv:
        assert c.qk_rope(cache=bad) == c.window(cache=bad, window=1) == c.prefix(cache=bad) == c.prefix(prefix=bad) == SHAPE, bad
    for bad in (dict(B=0), dict(T=0), dict(B=3), dict(Hq=0), dict(Hq=1025), dict(T=1 << 20), dict(rope=dict(rotary_dim=63)), dict(rope=dict(rotary_dim=130)),
                dict(rope=dict(rotary_dim=-2)), dict(q=dict(stride_t=-1024)), dict(T=9, cache=dict(ring=8))):
        assert c.qk_rope(**bad) == SHAPE, bad
    assert c.qk_rope(T=9, cache=dict(ring=8), slots=p) == WORKSPACE                     # the caller names the rows
    for bad in (dict(B=0), dict(T=0), dict(B=3), dict(Hq=3), dict(Hq=0), dict(B=4097, cache=dict(batch=5000)), dict(T=1 << 20), dict(out=dict(stride_h=-128))):
        assert c.window(**bad) == SHAPE, bad
    ring = dict(n_sink=4, ring=60)
    for bad in (dict(window=0), dict(window=61), dict(window=60, T=2), dict(window=60, sinks=5)):
        assert c.window(cache=ring, **bad) == SHAPE, bad
    for bad in (dict(n=0), dict(n=65), dict(B=3), dict(Hq=3), dict(prefix=dict(d=64)), dict(prefix=dict(heads=4)), dict(prefix=dict(dtype=b.F32))):
        assert c.prefix(**bad) == SHAPE, bad
    # types, alignment, scalars
    for t in (2, -1):
        assert c.qk_rope(cache=dict(dtype=t)) == c.window(cache=dict(dtype=t)) == c.prefix(cache=dict(dtype=t)) == DTYPE
    for bad in (dict(cache=dict(k=p + 8)), dict(cache=dict(stride_h=8190)), dict(q=dict(data=p + 2)), dict(q=dict(stride_h=132)), dict(out=dict(data=p + 8))):
        assert c.qk_rope(**bad) == c.window(**bad) == c.prefix(**bad) == ALIGN, bad
    assert c.qk_rope(pos=p + 2) == c.qk_rope(slots=p + 1) == c.qk_rope(rope=dict(turns=p + 8)) == c.qk_rope(norm=dict(q_weight=p + 2)) == ALIGN
    assert c.window(lens=p + 1) == c.window(q_lens=p + 2) == c.window(lse=p + 3) == c.prefix(lens=p + 1) == ALIGN
    nan, inf = float("nan"), float("inf")
    assert c.qk_rope(rope=dict(layout=2)) == c.qk_rope(rope=dict(magnitude=inf)) == c.qk_rope(norm=dict(eps=-1.0)) == c.qk_rope(norm=dict(offset=nan)) == VALUE
    assert c.window(window=-1) == c.window(sinks=-1) == c.window(scale=nan) == c.prefix(scale=inf) == VALUE
    assert c.prefix(cache=dict(ring=8)) == c.prefix(prefix=dict(ring=8)) == VALUE
    assert b"ring" in c.lib.clada_last_error(c.h)
    c.lib.clada_destroy(c.h)


def test_workspace_bound_grows_with_the_call(b):
    f = b.attn_workspace_bytes
    assert f(0, 1, 1, 1) == f(1, 1, 0, 128) == 256
    assert f(1, 1, 8, 128) < f(2, 1, 8, 128) < f(2, 1, 8, 256)
    assert f(4096, 1, 64, 256) < 1 << 31
    sizes = [1, 2, 5, 16, 64, 300, 4096]
    for d in (8, 128):                                       # a workspace for a call is one for every smaller call
        table = np.array([[[f(B, T, Hq, d) for Hq in sizes] for T in sizes] for B in sizes], float)
        assert all(np.all(np.diff(table, axis=k) >= 0) for k in range(3))


@pytest.mark.parametrize("kind", ["none", "linear", "base", "bands", "ramp"])
@pytest.mark.parametrize("R", [2, 24, 64, 80, 128, 256])
@pytest.mark.parametrize("theta", [10000.0, 500000.0, 1.5])
def test_turns_are_the_frequencies(b, kind, R, theta):
    """A frequency of a few units of 2^-53, as a 64-bit fraction of a turn truncated to 2^-64."""
    c = Calls(b)
    turns, m = np.zeros(R // 2, np.uint64), C.c_float()
    s = b._CRopeScaling(theta, 8.0, 4096.0, 1.0, 4.0, ["none", "linear", "base", "bands", "ramp"].index(kind))
    assert c.lib.clada_rope_turns(c.h, R, C.byref(s), turns.ctypes.data, C.byref(m)) == OK
    f, mag = ref.frequencies(R, theta, kind)
    assert np.allclose(turns.astype(np.float64) / 2.0 ** 64 * (2 * np.pi), f, rtol=1e-13, atol=2.0 ** -60) and abs(m.value - mag) < 1e-6
    for bad in (dict(theta=0.5), dict(theta=float("inf")), dict(kind=5), dict(kind=-1), dict(kind=1, factor=0.5), dict(kind=3, low=4.0), dict(kind=4, original_len=0.0),
                dict(kind=4, theta=1.0), dict(kind=3, high=float("nan"))):
        t = b._CRopeScaling(**{**dict(theta=theta, factor=8.0, original_len=4096.0, low=1.0, high=4.0, kind=1), **bad})
        assert c.lib.clada_rope_turns(c.h, R, C.byref(t), turns.ctypes.data, C.byref(m)) == VALUE, bad
    for r in (0, 1, 3, 258, -2):
        assert c.lib.clada_rope_turns(c.h, r, C.byref(s), turns.ctypes.data, C.byref(m)) == SHAPE
    assert c.lib.clada_rope_turns(c.h, R, None, turns.ctypes.data, C.byref(m)) == NULL
    c.lib.clada_destroy(c.h)


def test_the_binding_refuses_host_tensors(b):
    with pytest.raises(AssertionError):
        b.KVCache(torch.zeros(1, 1, 4, 64), torch.zeros(1, 1, 4, 64))


def test_outputs_on_top_of_each_other_are_refused(b):
    """A stride of 0, or below the values of a head, along a dimension of more than one: for outputs and for what is stored, not for inputs."""
    c = Calls(b)
    low = dict(stride_b=0), dict(stride_t=64), dict(stride_h=0), dict(stride_h=120)
    for s in low:
        assert c.qk_rope(out=s) == c.window(out=s, T=3) == SHAPE, s
        assert c.qk_rope(q=s, k=s, v=s) == c.window(q=s, T=3) == c.prefix(q=s) == WORKSPACE, s
    assert c.window(out=low[0]) == SHAPE and b"on top of each other" in c.lib.clada_last_error(c.h)
    for s in (low[0], low[2], low[3]):
        assert c.prefix(out=s) == SHAPE, s
    # a dimension of one row has no stride to speak of
    assert c.window(out=dict(stride_b=0, stride_t=0, stride_h=0), B=1, T=1, Hq=1, cache=dict(heads=1)) == WORKSPACE
    assert c.window(out=dict(stride_t=0)) == c.prefix(out=dict(stride_t=0)) == WORKSPACE
    assert c.qk_rope(out=dict(stride_b=0, stride_t=0, stride_h=0), B=1, T=1, Hq=1) == WORKSPACE
    # the cache: read with any strides, stored into with rows and heads of their own
    for s in (dict(stride_h=0), dict(stride_h=64), dict(stride_n=0), dict(stride_n=64)):
        assert c.qk_rope(cache=s) == SHAPE and c.qk_rope(cache=s, k=None, v=None) == c.window(cache=s) == c.prefix(cache=s) == c.prefix(prefix=s) == WORKSPACE, s
    assert c.qk_rope(cache=dict(stride_b=0), slots=c.p) == c.qk_rope(cache=dict(stride_n=0), T=1) == c.qk_rope(cache=dict(stride_n=0, capacity=1)) == WORKSPACE
    c.lib.clada_destroy(c.h)
