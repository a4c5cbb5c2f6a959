"""Scales and caps that the attention calls cannot form scores with in base 2 (times log2(e), 1.4427) are refused on the host (CPU only)."""
import test_attention_abi as contiguous
import test_paged_abi as paged
from test_paged_abi import VALUE, WORKSPACE, b  # noqa: F401 (fixture)

MOST = 3.4028234663852886e38 / 1.4426950408889634                  # 2.3586e38


def test_scales_beyond_fp32_in_base_2(b):
    c, p = contiguous.Calls(b), paged.Calls(b)
    for scale in (MOST * (1 - 1e-6), -MOST * (1 - 1e-6), 1e38, 0.0, 1e-45):
        assert c.window(scale=scale) == c.prefix(scale=scale) == p.attn(scores=dict(scale=scale)) == WORKSPACE, scale       # accepted up to the missing device
    for scale in (MOST * (1 + 1e-6), -3e38, 3.4e38):
        assert c.window(scale=scale) == c.prefix(scale=scale) == p.attn(scores=dict(scale=scale)) == VALUE, scale
    c.lib.clada_destroy(c.h)
    p.lib.clada_destroy(p.h)


def test_caps_beyond_fp32_in_base_2(b):
    c = paged.Calls(b)
    # a cap takes the scale in: only its own size counts; one of 2^100 |scale| or more, or beside a scale of 0, is none
    for cap, scale in ((MOST * (1 - 1e-6), 1e38), (1.0, 3.4e38), (1e-45, -3.4e38), (3.4e38, 1e8), (3.4e38, 0.0), (3.4e38, 1e-45), (3e38, 0.125)):
        assert c.attn(scores=dict(cap=cap, scale=scale)) == WORKSPACE, (cap, scale)
    for cap, scale in ((MOST * (1 + 1e-6), 1e38), (3.4e38, -1e9), (3.4e38, 3.4e38)):
        assert c.attn(scores=dict(cap=cap, scale=scale)) == VALUE, (cap, scale)
    assert b"cap" in c.lib.clada_last_error(c.h)
    c.lib.clada_destroy(c.h)
