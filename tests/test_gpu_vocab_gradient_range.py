"""dW of words whose gradients are far below the others': unlikely in every row, in the rows of some tiles only, or known to rows of small dloss only.

Tolerances: those of test_gpu_vocab_loss.py (from there: ez, e_lse, exp, sums), but each word by itself.  u = 2^-24.
  dz   p times (ez + e_lse + exponential) and three roundings of dz; where it is not a label's, p - 0 has no error of its own.  fp16: one plane (bf16
       gradients) rounds it by 2^-11, two (f32 gradients) by 2^-22.
  dW   in fp16 a word's largest |dz| stands at 2^-4 or above, in steps of 2^-24: a value is off by up to 2^-25 where its tile rounds it and by as much
       again where the word's tiles are brought together, 2^-20 of the word's largest; two planes have 2^-11 of that.
"""
import numpy as np
import pytest

from oracle import vocab_ref as vr
from test_gpu_vocab_loss import Problem, U

pytestmark = pytest.mark.gpu

RARE = {3: 14.0, 40: 20.0, 41: 24.0, 77: 28.0, 130: 40.0, 200: 60.0}   # word: how far its logit is lowered in all rows
FIRST, LAST, SMALL = (5, 90, 129), (6, 91), (7, 92, 201)               # in the first rows, in the last rows; for the rows of large dloss


def _problem(N, V, D, out, small):
    import torch
    p = Problem(N, V, D, "bf16", out, 0.0, pad=0.1, seed=N + D)
    special = [*RARE, *FIRST, *LAST, *SMALL]
    p.labels[np.isin(p.labels, special)] = 300
    h, W, rows = p.h.float().numpy(), p.W.float().numpy(), np.arange(N)
    h[:, :4] = 0.0
    W[:, :4] = 0.0
    h[:, 0] = 4.0
    for v, down in RARE.items():
        W[v, 0] = -down / 4.0
    cut = min(N // 2, 260)
    h[rows < cut, 1], h[rows >= cut, 2] = 4.0, 4.0
    W[list(FIRST), 1] = W[list(LAST), 2] = -7.0
    p.dloss = torch.full((N,), 1.0 / N)
    if small:
        p.dloss *= torch.exp2(-torch.from_numpy(rows % 3 * 10).float())
        h[rows % 3 != 2, 3] = 4.0
        W[list(SMALL), 3] = -9.0
    p.h, p.W = torch.from_numpy(h).bfloat16(), torch.from_numpy(W).bfloat16()
    return p


@pytest.mark.parametrize("small", [False, True], ids=["equal_dloss", "small_dloss"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
# one row tile; several of 128; several of 256; sums in parts; many row tiles and two pieces of the vocabulary
@pytest.mark.parametrize("N,V,D", [(100, 700, 72), (700, 1500, 136), (1000, 9001, 520), (5000, 400, 64), (9000, 8300, 40)])
def test_words_with_nothing_but_small_gradients(N, V, D, out, small):
    p = _problem(N, V, D, out, small)
    got = p.run(want_dh=False)["dW"]
    h, W, g = p.h.double().numpy(), p.W.double().numpy(), np.abs(p.dloss.double().numpy())
    rows = vr.labelled(p.labels, V)
    h, g = h[rows], g[rows]
    z = h @ W.T
    lse = vr.loss_forward(p.h.double().numpy(), W, p.labels, 0.0)[1][rows, None]
    prob = np.exp(z - lse)
    label = np.arange(V) == p.labels[rows, None]
    dz = g[:, None] * (prob - label)
    ez = (4 * -(-D // 16) + 4) * U * (np.abs(h) @ np.abs(W).T)
    span = np.minimum(2 + 2 * (z.max(1) - z.min(1)), 220)
    e_lse = ez.max(1) + (span + V / 64 + 80) * U + 3 * U * (np.abs(lse[:, 0]) + np.abs(z).max(1) + 1)
    planes = 1 if out == "bf16" else 2
    e_dz = g[:, None] * (prob * (ez + e_lse[:, None] + (4 + 2 * np.abs(z - lse)) * U) + 3 * U * label) + (3 * U + 2.0 ** (-11 * planes)) * np.abs(dz)
    ref, size = dz.T @ h, np.abs(dz).T @ np.abs(h)
    bound = e_dz.T @ np.abs(h) + 2.0 ** (-9 - 11 * planes) * np.abs(dz).max(0)[:, None] * np.abs(h).sum(0)
    bound += (4 * planes * (len(rows) // 16 + 4) + 8) * U * size + (2.0 ** -8 if out == "bf16" else U) * np.abs(ref)
    bound += 2.0 ** -40 * np.abs(dz).sum(0)[:, None] * np.abs(h).max()                 # h, scaled to at least 2^15
    worse = np.flatnonzero((np.abs(got - ref) > 1.01 * bound).any(1))
    norm = np.linalg.norm
    print("worst words", {int(v): "%.2g" % (norm(got[v] - ref[v]) / norm(ref[v])) for v in worse[:12]}, flush=True)
    assert len(worse) == 0
