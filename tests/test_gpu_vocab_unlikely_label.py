"""Rows whose label is far less likely than other words, down to a logit of minus infinity: lse does not depend on the label's logit then.

Tolerance of lse: the other words' logits have the errors ez of test_gpu_vocab_loss.py (the label's own is not part of their sum), the exponentials and
the sum (2 + 2 span + V / 64 + 80) u, logarithm and two sums 3 u of the size of lse; u = 2^-24."""
import numpy as np
import pytest

from test_gpu_vocab_loss import Problem, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [64.0, 4096.0, 2.0 ** 20])
@pytest.mark.parametrize("store", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,D", [(1, 500, 64), (40, 500, 64), (1300, 2500, 130)])
def test_lse_of_an_unlikely_label(N, V, D, store, far):
    p = Problem(N, V, D, store, "f32", 0.0, pad=0.0, seed=N + 1)
    p.h[:, 0], p.W[:, 0] = 1.0, 0.0
    p.labels[:] = np.arange(N) % 7
    p.W[:7, 0] = -far
    got = p.run()
    h, W = p.h.double().numpy(), p.W.double().numpy()
    z = h @ W.T
    others = z[:, 7:]
    top = others.max(1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(1))
    S = (6 if store == "f32" else 1) * -(-D // 16)
    ez = ((4 * S + 4) * U * (np.abs(h) @ np.abs(W[7:]).T)).max(1)
    e = ez + (2 + 2 * np.minimum(others.max(1) - others.min(1), 110) + V / 64 + 80) * U + 3 * U * (np.abs(lse) + 1)
    assert (np.abs(got["lse"] - lse) <= e).all(), np.abs(got["lse"] - lse).max()
    zy = z[np.arange(N), p.labels]
    ezy = (4 * S + 4) * U * (np.abs(h) * np.abs(W[p.labels])).sum(1)
    assert (np.abs(got["loss"] - (lse - zy)) <= e + ezy + 3 * U * np.abs(lse - zy)).all()


@pytest.mark.parametrize("N,V,D", [(1, 500, 64), (40, 500, 64), (1300, 2500, 136)])
def test_a_label_of_minus_infinity(N, V, D):
    """Its loss is infinite; lse, and what the other words' rows of dW get, are what a label far below gives."""
    p = Problem(N, V, D, "bf16", "f32", 0.0, pad=0.0, seed=N + 2)
    p.h = p.h.abs() + 0.125                                # positive: z = -inf, not NaN
    p.labels[:] = np.arange(N) % 7
    p.W[:7] = -1e6
    want = p.run(want_dh=False)
    p.W[:7] = -np.inf
    got = p.run(want_dh=False)
    assert (got["loss"] == np.inf).all()
    assert np.array_equal(got["lse"], want["lse"]) and np.array_equal(got["dW"], want["dW"])


@pytest.mark.parametrize("N,V,D", [(1, 500, 64), (40, 500, 64), (1300, 2500, 136)])
def test_a_label_of_infinity_is_no_loss_of_zero(N, V, D):
    """The difference of two infinities, as for any other word's."""
    p = Problem(N, V, D, "bf16", "f32", 0.0, pad=0.0, seed=N + 3)
    p.h = p.h.abs() + 0.125
    p.labels[:] = 3
    p.W[3] = np.inf
    got = p.run(forward_only=True)
    assert np.isnan(got["loss"]).all() and not np.isfinite(got["lse"]).any()
