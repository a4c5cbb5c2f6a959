"""What the paged cache's calls rest on outside the kernels (CPU only): the binding's packed structs, and the reference for long prompts."""
import ctypes as C
import os

import numpy as np
import pytest

import paged_dense as dense
import paged_ref as paged


@pytest.fixture(scope="module")
def b():
    import paper_2502_19078_amd as pkg
    if not os.path.exists(pkg.lib_path()):
        from paper_2502_19078_amd import build
        build.build()
    import paper_2502_19078_amd.binding as binding
    return binding


@pytest.mark.parametrize("pack,cls", [("_PACK_HEADS", "_CHeads"), ("_PACK_ROPE", "_CRope"), ("_PACK_NORM", "_CHeadNorm"), ("_PACK_PAGED", "_CPagedCache"),
                                      ("_PACK_SCORES", "_CAttnScores")])
def test_packed_structs_are_those_of_the_classes(b, pack, cls):
    """Every field, packed by itself beside zeros, is where the ctypes class has it, and the size is the class's."""
    pack, cls = getattr(b, pack), getattr(b, cls)
    zeros = [0] * len(cls._fields_)
    assert len(pack(*zeros)) == C.sizeof(cls)
    for i, (name, kind) in enumerate(cls._fields_):
        value = 1.5 if kind is C.c_float else 3
        s = cls.from_buffer_copy(pack(*zeros[:i], value, *zeros[i + 1:]))
        assert [getattr(s, n) or 0 for n, _ in cls._fields_] == zeros[:i] + [value] + zeros[i + 1:], name


@pytest.mark.parametrize("kw", [dict(), dict(window=9, cap=1.5), dict(cap=3.0, slopes=[0.1, 0.0, 0.5, 1.0]), dict(slopes=[0.1, 0.0, 0.5, 1.0], fp32=True, cap=2.0)])
def test_the_reference_for_long_prompts_is_the_plain_one(kw):
    rng = np.random.default_rng(1)
    T, n, d, page, table = 9, 40, 8, 16, [2, 0, 1]
    q, k, v = rng.standard_normal((1, T, 4, d)), rng.standard_normal((3, 2, page, d)), rng.standard_normal((3, 2, page, d))
    a = dense.paged_attn(q, k, v, table, page, n, 0.4, **kw)
    w = paged.paged_attn(q, k, v, [table], page, [n], [T], 0.4, **kw)
    for key in w:
        assert np.allclose(a[key], w[key], rtol=1e-12, atol=1e-13), key
