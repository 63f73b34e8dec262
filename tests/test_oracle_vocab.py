"""The vocabulary oracle itself: gradients against central differences, the loss against its definition written per word, invariants."""
import numpy as np
import pytest

from oracle import vocab_ref as vr


def _inputs(N, V, D, seed, scale=1.0):
    r = np.random.default_rng(seed)
    h, W = scale * r.standard_normal((N, D)), r.standard_normal((V, D)) / np.sqrt(D)
    labels = r.integers(0, V, N)
    labels[::4] = -1
    return h, W, labels, r.standard_normal(N)


@pytest.mark.parametrize("eps", [0.0, 0.1, 0.5])
def test_loss_is_the_cross_entropy_with_the_smoothed_target(eps):
    h, W, labels, _ = _inputs(7, 11, 5, 0)
    loss, lse = vr.loss_forward(h, W, labels, eps)
    for n in range(7):
        if labels[n] < 0:
            assert loss[n] == 0 and lse[n] == 0
            continue
        z = [sum(h[n, d] * W[v, d] for d in range(5)) for v in range(11)]
        log_p = [x - np.log(sum(np.exp(y) for y in z)) for x in z]
        target = [eps / 11 + (1 - eps) * (v == labels[n]) for v in range(11)]
        assert abs(loss[n] + sum(t * l for t, l in zip(target, log_p))) < 1e-12


@pytest.mark.parametrize("eps", [0.0, 0.1])
def test_loss_gradients_are_the_differences(eps):
    h, W, labels, dloss = _inputs(5, 7, 3, 1)
    dh, dW, _ = vr.loss_backward(dloss, h, W, labels, eps)
    step = 1e-5
    for x, dx in ((h, dh), (W, dW)):
        for i in np.ndindex(x.shape):
            keep = x[i]
            f = []
            for s in (step, -step):
                x[i] = keep + s
                f.append((dloss * vr.loss_forward(h, W, labels, eps)[0]).sum())
            x[i] = keep
            assert abs((f[0] - f[1]) / (2 * step) - dx[i]) < 1e-8


def test_dz_of_a_row_sums_to_zero():
    h, W, labels, dloss = _inputs(9, 13, 4, 2)
    assert np.abs(vr.loss_backward(dloss, h, W, labels, 0.1)[2].sum(1)).max() < 1e-14


def test_embedding_gradient_is_the_transposed_map():
    """<embed(E), g> = <E, embed'(g)> for every E, g: the map is linear."""
    r = np.random.default_rng(3)
    tokens = np.array([3, 0, 3, -1, 9, 3, 5, 100])
    E, g = r.standard_normal((9, 4)), r.standard_normal((8, 4))
    out = vr.embed_forward(tokens, E, 1.7)
    back, _ = vr.embed_backward(tokens, g, 1.7, 9)
    assert abs((out * g).sum() - (E * back).sum()) < 1e-12
    assert not out[[3, 4, 7]].any()


def test_clipping():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    assert vr.grad_norm(g) == 5.0
    assert np.allclose(vr.grad_clip(g, 1.0)[1][0], [0.6, 0.0])
    assert vr.grad_clip(g, 5.0)[1][0][0] == 3.0
    assert vr.grad_clip([np.array([np.inf, 1.0])], 1.0)[1][0][1] == 1.0
