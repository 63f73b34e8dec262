"""The distillation's loss where student and teacher are nearly sure of the same word: a small number, which keeps its digits.

Logits are exact here (a row's word has s, all others 0), so the loss has a closed form.  With n = K - 1 other entries of logit 0 beside the word's t, a = s / T, b = t / T:
  loss / T^2 = log(1 + (V - 1) e^-a) - log(1 + n e^-b) + n q (a - b)        q = e^-b / (1 + n e^-b), the share of one of them
Tolerance, u = 2^-24: the kernels add and subtract the terms  log(1 + (V - 1) e^-a),  log(1 + n e^-b),  n q a  and  n q b, each of them with an error in parts of itself:
an exponential's argument is rounded twice or three times (3 a u, 3 b u), it is good to 2 u, sums have the roundings of test_gpu_distill.py (V / 64 + 80 and K), the
logarithm, the products and T^2 below 12 u.  So the error is at most  T^2 (3 (a + b) + V / 64 + K + 100) u  times the sum of the four."""
import numpy as np
import pytest

from test_gpu_distill import Problem
from test_gpu_scan import U, _torch

pytestmark = pytest.mark.gpu


def _sure(N, V, K, T, store, seed, top_at=0):
    """Row n: word 37 (n % 16) + 5 has s[n], the teacher's list it with t[n] at place top_at and K - 1 other words with 0."""
    torch, _, types = _torch()
    D, p, r = 64, Problem(N, V, 64, K, store, T=T, pad=0.0, seed=seed), np.random.default_rng(seed)
    own = 37 * (np.arange(N) % 16) + 5
    s, t = np.round(T * (12 + 20 * r.random(N)) * 4) / 4, np.round(T * (10 + 20 * r.random(N)) * 4) / 4
    W, h = np.zeros((V, D), np.float32), np.zeros((N, D), np.float32)
    W[37 * np.arange(16) + 5, np.arange(16)] = 1.0
    h[np.arange(N), np.arange(N) % 16] = s
    words, logits = np.zeros((N, K), np.int32), np.zeros((N, K), np.float32)
    for n in range(N):
        others = r.choice(np.delete(np.arange(V), 37 * np.arange(16) + 5), K - 1, replace=False)
        words[n] = np.insert(others, top_at, own[n])
        logits[n, top_at] = t[n]
    p.words, p.logits = words, torch.from_numpy(logits)
    p.h, p.W = torch.from_numpy(h).to(types[store]), torch.from_numpy(W).to(types[store])
    assert (p.h.double().numpy() == h).all()
    return p, s / T, t / T


@pytest.mark.parametrize("N", [1, 5, 16, 40, 64, 130, 700])
@pytest.mark.parametrize("V", [700, 5003])
@pytest.mark.parametrize("store", ["f32", "bf16"])
@pytest.mark.parametrize("K,T,top_at", [(1, 1.0, 0), (10, 1.0, 0), (10, 2.0, 7), (100, 1.0, 99)])
def test_a_sure_teacher_and_a_sure_student(N, V, store, K, T, top_at):
    p, a, b = _sure(N, V, K, T, store, seed=N + V + K, top_at=top_at)
    got = p.run(forward_only=True)
    n = K - 1
    q = np.exp(-b) / (1 + n * np.exp(-b))
    terms = np.log1p((V - 1) * np.exp(-a)), np.log1p(n * np.exp(-b)), n * q * a, n * q * b
    want = T * T * (terms[0] - terms[1] + terms[2] - terms[3])
    bound = T * T * (3 * (a + b) + V / 64 + K + 100) * U * sum(terms)
    assert (np.abs(got["loss"] - want) <= bound).all(), (np.abs(got["loss"] - want) / bound).max()
    p.check(got)


@pytest.mark.parametrize("N,V", [(1, 1), (3, 1), (5, 700), (40, 129), (64, 5000), (300, 5003), (700, 131)])
@pytest.mark.parametrize("store", ["f32", "bf16"])
def test_logits_that_are_all_the_same(N, V, store):
    """Every word is a likeliest one: lse = log V + z."""
    torch, _, types = _torch()
    p = Problem(N, V, 32, 3, store, pad=0.0, seed=N)
    p.h, p.W = torch.zeros(N, 32).to(types[store]), torch.zeros(V, 32).to(types[store])
    p.h[:, 0], p.W[:, 0] = torch.arange(N).to(types[store]) / 8, 1.0
    p.words[:, 0], p.logits[:, 0] = V - 1, 0.5
    got = p.run()
    z = p.h[:, 0].double().numpy()
    assert (np.abs(got["lse"] - z - np.log(V)) <= (V / 64 + 80) * U + 3 * U * (z + np.log(V) + 1)).all()
    p.check(got)
