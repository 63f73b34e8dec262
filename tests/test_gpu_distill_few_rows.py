"""Few f32 rows of the distillation: the small parts of a logit are summed by themselves.

A logit whose products' large parts add up to about 2^14 without any rounding (whole numbers), and whose small parts are 0.4 steps of that sum for every 32
numbers: added to it one after the other they would all be lost, 2 D / 160 steps.  What remains, u = 2^-24: the small sum's own roundings, D / 32 of u of
itself (64 of at most 2^-4: far below a step), one rounding where it is added and one each of the logarithm's and lse's: 4 steps of lse at most."""
import numpy as np
import pytest

from test_gpu_distill import Problem
from test_gpu_scan import _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 16, 17, 32, 33, 64, 100])
def test_small_parts_are_not_lost(N):
    torch, _, _ = _torch()
    V, D = 130, 2048
    p = Problem(N, V, D, 1, "f32", pad=0.0, seed=N)
    small = 1.6 * 2.0 ** -16                                  # 32 of them: 0.4 steps of a number in 2^14 .. 2^15
    h, W = np.ones((N, D)), np.zeros((V, D))
    h[:, 0] = 128
    W[7], W[100] = 1 + small, -1.0
    W[7, 0] = 128
    p.h, p.W = torch.from_numpy(h.astype(np.float32)), torch.from_numpy(W.astype(np.float32))
    p.words[:, 0], p.logits[:, 0] = 7, 1.0
    got = p.run()
    lse = (p.h.double() @ p.W.double().T)[:, 7].numpy()       # the others are 0 and less: e^-18000
    step = 2.0 ** (14 - 23)
    assert (2 ** 14 < lse).all() and (lse < 2 ** 15).all()
    assert (np.abs(got["lse"] - lse) <= 4 * step).all(), np.abs(got["lse"] - lse).max() / step
    p.check(got)
