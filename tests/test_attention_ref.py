"""That the bounds of attention_ref.py tell the precisions apart that the header promises: weights rounded to one bf16 in the oracle stay within the
bound of one bf16 and leave that of two; weights rounded to 16 bits stay within that.  CPU only."""
import numpy as np
import pytest

import attention_ref as ref
import synth


def _bf16(x):
    return synth.bf16_widen(synth.bf16_bits(np.asarray(x, np.float32))).astype(np.float64)


@pytest.mark.parametrize("n", [20, 130, 500])
def test_one_bf16_of_a_weight_is_not_two(n):
    rng = np.random.default_rng(n)
    d, rows = 64, 6
    q, k, v = (_bf16(rng.standard_normal((m, d))) for m in (rows, n, n))
    r = dict(out=np.zeros((rows, d)), lse=np.zeros(rows), mag=np.zeros((rows, d)), S=np.zeros(rows), n=np.full(rows, n))
    one, two = np.zeros((rows, d)), np.zeros((rows, d))
    for i in range(rows):
        r["out"][i], r["lse"][i], r["mag"][i], r["S"][i] = ref.attend(q[i], k, v, d ** -0.5)
        s = d ** -0.5 * (k @ q[i])
        w = np.exp(s - s.max())
        hi = _bf16(w)
        one[i], two[i] = hi @ v / w.sum(), (hi + _bf16(w - hi)) @ v / w.sum()
    one, two = _bf16(one), _bf16(two)
    ref.check(two, r["lse"], r, "bf16")
    ref.check(one, r["lse"], r, "bf16", weights_bf16=True)
    with pytest.raises(AssertionError, match="more than the bound"):
        ref.check(one, r["lse"], r, "bf16")
