"""The float64 definitions of the recurrence, the distillation and the verification against differences, invariants and counting."""
import numpy as np
import pytest

from oracle import student_ref as sr
from oracle import vocab_ref as vr


def _scan_inputs(B, T, H, seed):
    r = np.random.default_rng(seed)
    return r.standard_normal((B, T, 3 * H)), r.standard_normal((B, H)), r.standard_normal((B, T, H)), r.standard_normal((B, H))


@pytest.mark.parametrize("reverse", [False, True])
def test_scan_gradients_against_differences(reverse):
    B, T, H, n = 3, 5, 2, np.array([5, 0, 3])
    G, c0, dh, dc = _scan_inputs(B, T, H, 1)
    f = lambda: (lambda h, c: (dh * h).sum() + (dc * c).sum())(*sr.scan_forward(G, c0, n, reverse))
    dG, dc0 = sr.scan_backward(dh, dc, G, c0, n, reverse)
    for x, grad in ((G, dG), (c0, dc0)):
        for at in np.ndindex(x.shape):
            old = x[at]
            x[at] = old + 1e-5
            up = f()
            x[at] = old - 1e-5
            down = f()
            x[at] = old
            assert abs((up - down) / 2e-5 - grad[at]) < 1e-8
    assert (dG[1] == 0).all() and (dc0[1] == dc[1]).all() and (dG[2, 3:] == 0).all()


def test_scan_runs_backwards_as_forwards():
    G, c0, *_ = _scan_inputs(2, 6, 3, 2)
    n = np.array([6, 4])
    h, c = sr.scan_forward(G, c0, n, True)
    for b in range(2):
        turned, last = sr.scan_forward(G[b:b + 1, :n[b]][:, ::-1], c0[b:b + 1], None)
        assert np.array_equal(h[b, :n[b]], turned[0, ::-1]) and np.array_equal(c[b], last[0])


def test_distillation_gradients_against_differences():
    r = np.random.default_rng(3)
    N, V, D, K, T = 4, 7, 3, 5, 1.7
    h, W, t, g = r.standard_normal((N, D)), r.standard_normal((V, D)), r.standard_normal((N, K)), r.standard_normal(N)
    words = r.integers(-1, V + 1, (N, K))
    words[0] = [2, 2, 5, 2, 1]                            # a word three times
    words[3] = -1
    t[1, 2] = -np.inf
    dh, dW, _ = sr.distill_backward(g, h, W, words, t, T)
    for x, grad in ((h, dh), (W, dW)):
        for at in np.ndindex(x.shape):
            old = x[at]
            x[at] = old + 1e-5
            up = (g * sr.distill_forward(h, W, words, t, T)[0]).sum()
            x[at] = old - 1e-5
            down = (g * sr.distill_forward(h, W, words, t, T)[0]).sum()
            x[at] = old
            assert abs((up - down) / 2e-5 - grad[at]) < 1e-8
    assert (dh[3] == 0).all()


def test_distillation_of_one_word_is_the_loss_of_its_label():
    r = np.random.default_rng(4)
    h, W, y = r.standard_normal((6, 4)), r.standard_normal((9, 4)), np.array([3, -1, 8, 0, 9, 5])
    a, b = sr.distill_forward(h, W, y[:, None], r.standard_normal((6, 1)), 1.0), vr.loss_forward(h, W, y, 0.0)
    assert np.allclose(a, b, rtol=0, atol=1e-13)
    ones = np.ones(6)
    for x, y_ in zip(sr.distill_backward(ones, h, W, y[:, None], np.zeros((6, 1)), 1.0)[:2], vr.loss_backward(ones, h, W, y, 0.0)[:2]):
        assert np.allclose(x, y_, rtol=0, atol=1e-13)


def test_verified_words_are_distributed_as_the_target():
    """Every choice of the drafted word and of a grid of u and r, with the weights that they have: the first word's distribution is p."""
    r = np.random.default_rng(5)
    V, grid = 5, 200
    p, q = r.dirichlet(np.ones(V)), r.dirichlet(np.ones(V))
    first = np.zeros(V)
    x = (np.arange(grid) + 0.5) / grid
    for d in range(V):
        u, v = (a.reshape(-1) for a in np.meshgrid(x, x))
        n = len(u)
        tokens, taken = sr.draft_verify(np.full((n, 1), d), None, np.broadcast_to(q, (n, 1, V)), np.broadcast_to(np.stack([p, p]), (n, 2, V)),
                                        u[:, None], v)
        assert ((taken == 1) == (u * q[d] < p[d])).all()
        np.add.at(first, tokens[:, 0], q[d] / n)
    assert np.abs(first - p).max() < 2.0 / grid


def test_verification_at_its_edges():
    p = np.array([[[0.5, 0.0, 0.25, 0.25], [0.0, 0.0, 0.0, 0.0], [np.nan, np.inf, -1.0, 2.0]]])
    q = np.array([[[0.5, 0.0, 0.25, 0.25], [0.25, 0.25, 0.25, 0.25]]])
    go = lambda d, u, r, n=None: [x.tolist() for x in sr.draft_verify(np.array([d]), n, q, p, np.array([u]), np.array([r]))]
    assert go([1, 0], [0.0, 0.0], 0.5) == [[[2, -1, -1]], [0]]               # 0 < 0 is false; nothing is left of p - q: p; 0.5 is not above 0.5
    assert go([1, 0], [0.0, 0.0], 0.49) == [[[0, -1, -1]], [0]]
    assert go([0, 0], [0.9, 0.0], 0.0) == [[[0, -1, -1]], [1]]               # no word to draw
    assert go([0, 4], [0.9, 0.0], 0.0, [1]) == [[[0, -1, -1]], [1]]
    assert go([7, 0], [0.0, 0.0], 1.0) == [[[3, -1, -1]], [0]]               # no word of the vocabulary; r of 1: the last one
    p[0, 1] = p[0, 2]
    assert go([0, 3], [0.0, 1.0], np.nan) == [[[0, 3, 3]], [2]]              # NaN, infinities and what is below zero are no weights
