"""Words whose every logit is minus infinity, from bf16 storage: probability zero, in labelled rows as behind the last of them."""
import numpy as np
import pytest

from test_gpu_vocab_loss import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,D", [(20, 300, 64), (141, 700, 72), (1003, 9001, 136)])
def test_words_of_minus_infinity_have_no_gradient(N, V, D, out):
    """Bit for bit what words so far down that exp() of them is zero give.  (dh is not formed: zero times an infinite word is none.)"""
    p = Problem(N, V, D, "bf16", out, 0.0, pad=0.3, seed=N)
    p.h = p.h.abs() + 0.125                                # positive: z = -inf, not NaN
    down = [5, 130, V - 1]
    p.labels[np.isin(p.labels, down)] = 0
    p.W[down] = -1e6
    want = p.run(want_dh=False)
    p.W[down] = -np.inf
    got = p.run(want_dh=False)
    assert not got["dW"][down].any()
    for k in want:
        assert np.array_equal(got[k], want[k]), k
