"""CPU-only checks of the paged cache's calls: what they refuse, with which status, before any GPU is touched, and what the binding refuses
by itself."""
import ctypes as C
import os

import pytest
import torch

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
        self.p = p = (C.addressof(self.buf) + 255) // 256 * 256
        self.heads = dict(data=p, stride_b=4096, stride_t=1024, stride_h=128)
        self.paged = dict(k=p, v=p, k_scales=p, v_scales=p, stride_p=4096, stride_h=2048, stride_n=128, table=p, table_stride=4, pages=9, heads=2, page_size=16, d=128,
                          batch=2, max_pages=4, type=b.PAGE_BF16)
        self.rope = dict(turns=p, rotary_dim=64, layout=0, magnitude=1.0)
        self.scores = dict(scale=1.0, cap=0.0, slopes=None, prefix_lens=None, first=None, window=0)

    def _s(self, cls, base, change):
        return None if change is None else C.byref(cls(**{**base, **change}))

    def append(self, q={}, k={}, v={}, out={}, cache={}, rope={}, norm=None, B=2, T=3, Hq=4, pos=True):
        b, H = self.b, lambda x: self._s(b._CHeads, self.heads, x)
        n = None if norm is None else C.byref(b._CHeadNorm(**{**dict(q_weight=self.p, k_weight=self.p, eps=1e-6, offset=0.0), **norm}))
        return self.lib.clada_paged_rope(self.h, self._s(b._CRope, self.rope, rope), n, B, T, Hq, H(q), H(k), H(v), self.p if pos is True else pos, H(out),
                                         self._s(b._CPagedCache, self.paged, cache), None)

    def read(self, k={}, v={}, cache={}, pos=True, B=2, T=3):
        b, H = self.b, lambda x: self._s(b._CHeads, self.heads, x)
        return self.lib.clada_paged_read(self.h, self._s(b._CPagedCache, self.paged, cache), self.p if pos is True else pos, B, T, H(k), H(v), None)

    def attn(self, q={}, out={}, cache={}, lens=True, q_lens=None, B=2, T=1, Hq=4, max_len=0, scores={}, lse=None):
        b = self.b
        return self.lib.clada_paged_attn(self.h, self._s(b._CHeads, self.heads, q), self._s(b._CPagedCache, self.paged, cache), self.p if lens is True else lens, q_lens,
                                         B, T, Hq, max_len, self._s(b._CAttnScores, self.scores, scores), self._s(b._CHeads, self.heads, out), lse, None)


def test_refusals(b):
    c = Calls(b)
    p = c.p
    four = dict(type=b.PAGE_MX4)
    # accepted up to the missing device
    assert c.append() == c.append(norm={}) == c.append(q=None, out=None) == c.append(k=None, v=None) == c.append(cache=four) == WORKSPACE
    assert c.append(rope=dict(turns=None, rotary_dim=0)) == c.append(k=None, v=None, cache=dict(k=None, v=None, table=None)) == WORKSPACE
    assert c.append(cache=dict(pages=1, stride_p=0)) == c.append(cache=dict(heads=1, stride_h=0)) == WORKSPACE
    assert c.read() == c.read(k=None) == c.read(v=None) == c.read(cache=four) == c.read(cache=dict(k_scales=None, table_stride=0)) == WORKSPACE
    assert c.attn() == c.attn(T=9, q_lens=p, max_len=7, lse=p, scores=dict(cap=3.0, slopes=p, prefix_lens=p, first=p, window=5)) == c.attn(cache=four) == WORKSPACE
    assert c.attn(cache=dict(page_size=4096, stride_p=0, table_stride=7), q=dict(stride_h=0), scores=dict(scale=0.0)) == c.attn(scores=dict(scale=-1.0)) == WORKSPACE
    # no context, missing pointers
    assert c.lib.clada_paged_attn(None, None, None, None, None, 1, 1, 1, 0, None, None, None, None) == NULL
    assert c.lib.clada_paged_rope(None, None, None, 1, 1, 1, None, None, None, None, None, None, None) == NULL
    assert c.lib.clada_paged_read(None, None, None, 1, 1, None, None, None) == NULL
    for bad in (dict(q=None, k=None, v=None, out=None), dict(out=None), dict(v=None), dict(k=None), dict(pos=None), dict(cache=None), dict(rope=None),
                dict(q=dict(data=None)), dict(cache=dict(k=None)), dict(cache=dict(table=None)), dict(cache=dict(four, v_scales=None)), dict(rope=dict(turns=None))):
        assert c.append(**bad) == NULL, bad
    for bad in (dict(k=None, v=None), dict(pos=None), dict(cache=None), dict(k=dict(data=None)), dict(cache=dict(v=None)), dict(cache=dict(four, k_scales=None))):
        assert c.read(**bad) == NULL, bad
    for bad in (dict(q=None), dict(out=None), dict(cache=None), dict(lens=None), dict(scores=None), dict(cache=dict(v=None)), dict(cache=dict(table=None)),
                dict(cache=dict(four, k_scales=None)), dict(out=dict(data=None))):
        assert c.attn(**bad) == NULL, bad
    # sizes
    for bad in (dict(d=4), dict(d=100), dict(d=264), dict(four, d=80), dict(four, d=16), dict(batch=0), dict(heads=0), dict(heads=1025), dict(pages=0), dict(page_size=8),
                dict(page_size=24), dict(page_size=8192), dict(page_size=0), dict(page_size=-16), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(stride_n=-128),
                dict(stride_p=-4096), dict(table_stride=-1)):
        assert c.append(cache=bad) == c.attn(cache=bad) == c.read(cache=bad) == SHAPE, bad
    for bad in (dict(B=0), dict(T=0), dict(B=3), dict(Hq=0), dict(Hq=1025), dict(T=1 << 20), dict(rope=dict(rotary_dim=63)), dict(rope=dict(rotary_dim=130)),
                dict(q=dict(stride_t=-1024)), dict(cache=dict(stride_h=64)), dict(cache=dict(stride_n=0)), dict(cache=dict(stride_p=64)), dict(out=dict(stride_h=64))):
        assert c.append(**bad) == SHAPE, bad
    for bad in (dict(B=0), dict(T=0), dict(B=3), dict(T=1 << 20), dict(k=dict(stride_t=64)), dict(v=dict(stride_h=-128))):
        assert c.read(**bad) == SHAPE, bad
    for bad in (dict(B=0), dict(T=0), dict(B=3), dict(Hq=3), dict(Hq=0), dict(B=4097, cache=dict(batch=5000)), dict(T=1 << 20), dict(out=dict(stride_h=-128)),
                dict(out=dict(stride_b=64))):
        assert c.attn(**bad) == SHAPE, bad
    # types, alignment, scalars
    for t in (3, -1):
        assert c.append(cache=dict(type=t)) == c.attn(cache=dict(type=t)) == c.read(cache=dict(type=t)) == DTYPE
    for bad in (dict(k=p + 8), dict(stride_h=2052), dict(table=p + 2), dict(four, stride_n=136), dict(four, v=p + 8)):
        assert c.append(cache=bad) == c.attn(cache=bad) == c.read(cache=bad) == ALIGN, bad
    assert c.append(pos=p + 2) == c.append(rope=dict(turns=p + 8)) == c.append(q=dict(data=p + 2)) == c.read(pos=p + 1) == c.read(k=dict(data=p + 8)) == ALIGN
    for bad in (dict(lens=p + 1), dict(q_lens=p + 2), dict(lse=p + 3), dict(scores=dict(slopes=p + 1)), dict(scores=dict(prefix_lens=p + 2)),
                dict(scores=dict(first=p + 2)), dict(q=dict(stride_h=132))):
        assert c.attn(**bad) == ALIGN, bad
    nan, inf = float("nan"), float("inf")
    assert c.append(rope=dict(layout=2)) == c.append(rope=dict(magnitude=inf)) == c.append(norm=dict(eps=-1.0)) == VALUE
    for bad in (dict(max_len=-1), dict(scores=dict(scale=nan)), dict(scores=dict(scale=inf)), dict(scores=dict(cap=-1.0)), dict(scores=dict(cap=nan)),
                dict(scores=dict(cap=inf)), dict(scores=dict(window=-1))):
        assert c.attn(**bad) == VALUE, bad
    assert b"window" in c.lib.clada_last_error(c.h)
    c.lib.clada_destroy(c.h)


def test_the_binding_takes_tensors_on_the_gpu_alone(b):
    x, t = torch.zeros(4, 2, 16, 64), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(AssertionError):
        b.PagedCache(x, x, t)


def test_strides_that_the_kernels_do_not_reach(b):
    c = Calls(b)
    for most in (dict(stride_n=1 << 26, stride_h=1 << 31, stride_p=1 << 33), dict(stride_n=1 << 26, heads=1, pages=1)):
        assert c.read(cache=most) == c.attn(cache=most) == c.append(cache=most) == WORKSPACE
    for bad in (dict(stride_n=(1 << 26) + 32), dict(stride_p=(1 << 33) + 32), dict(stride_n=1 << 62), dict(stride_p=1 << 62)):
        assert c.read(cache=bad) == c.attn(cache=bad) == c.append(cache=bad) == SHAPE, bad
    c.lib.clada_destroy(c.h)
