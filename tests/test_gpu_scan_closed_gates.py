"""The recurrence behind gates that are nearly closed (f = sigmoid of -8 to -20): what passes such a gate, and its gradient, is small and keeps its digits.

Tolerances, for every value, from the arithmetic; u = 2^-24.  f and 1 - f are formed from e = 2^(-|x| log2 e), whose argument is rounded twice (2 |x| u, as
a part of e) and which is good to 2 u; one of them is 1 / (1 + e), good to 3 u, the other e times that: each is good to (2 |x| + 7) u OF ITS OWN, and so is a product of
several, to the sum of theirs.  All else as in test_gpu_scan.py; what is new against it is that every error of f is a part of f:
  c    behind candidates of zero:           E[t] = f E[t-1] + (2 |x| + 12) u f |c[t-1]|
  q    what a gate hands back, f r:         E[t] = f (E[t+1] + 16 u (ra + |dh|)) + (2 |x| + 12) u f ra
  dG   of the forget gate:                  f (1 - f) (E_r (ca + 1) + ra (E_c + 9 u) + (4 |x| + 24) u ra (ca + 1))"""
import numpy as np
import pytest

from oracle import student_ref as sr
from test_gpu_scan import HALF, Problem, U, _torch

pytestmark = pytest.mark.gpu

SIZES = [(3, 1, 12), (2, 3, 7), (3, 14, 70), (2, 50, 66), (2, 128, 9), (3, 200, 68), (2, 600, 64), (2, 600, 3)]


def _sigmoid(x):
    return 1 / (1 + np.exp(-x))


@pytest.mark.parametrize("B,T,H", SIZES)
@pytest.mark.parametrize("store,reverse", [("f32", False), ("f32", True), ("bf16", False)])
def test_gradients_of_closed_gates(B, T, H, store, reverse):
    torch, _, types = _torch()
    p = Problem(B, T, H, store, reverse, seed=B + T + H)
    r = np.random.default_rng(T)
    p.G[:, :, :H] = torch.from_numpy(np.where(r.random((B, T, H)) < 0.8, -8 - 12 * r.random((B, T, H)), 2 * r.standard_normal((B, T, H))).astype(np.float32)).to(types[store])
    got = p.run()
    G, dh, c0, dc = (x.double().numpy() for x in (p.G, p.dh, p.c0, p.dc_last))
    want_dG, want_dc0 = sr.scan_backward(dh, dc, G, c0, None, reverse)
    order = list(range(T - 1, -1, -1) if reverse else range(T))
    for b in range(B):
        x = np.abs(G[b, :, :H])
        f, k, g, o = _sigmoid(G[b, :, :H]), _sigmoid(-G[b, :, :H]), np.tanh(G[b, :, H:2 * H]), _sigmoid(G[b, :, 2 * H:])
        ca, E, before = np.abs(c0[b]), np.zeros(H), {}
        for t in order:
            before[t] = ca, E
            ca, E = f[t] * ca + k[t] * np.abs(g[t]), f[t] * E + 16 * U * (ca + 1)
        qa, E = np.abs(dc[b]), np.zeros(H)
        for t in reversed(order):
            ca, Ec = before[t]
            d = np.abs(dh[b, t])
            ra, Er = d * o[t] + qa, E + 16 * U * (d * o[t] + qa + d)
            bound = f[t] * k[t] * (Er * (ca + 1) + ra * (Ec + 9 * U) + (4 * x[t] + 24) * U * ra * (ca + 1)) + HALF[store] * np.abs(want_dG[b, t, :H])
            off = np.abs(got["dG"][b, t, :H] - want_dG[b, t, :H])
            assert (off <= 1.01 * bound + 2.0 ** -140).all(), (b, t, (off / bound).max())
            qa, E = f[t] * ra, f[t] * Er + (2 * x[t] + 12) * U * f[t] * ra
        off = np.abs(got["dc0"][b] - want_dc0[b])
        assert (off <= 1.01 * E + 2.0 ** -140).all(), (b, (off / E).max())
    p.check(got)


@pytest.mark.parametrize("B,T,H", SIZES)
@pytest.mark.parametrize("reverse", [False, True])
def test_what_closed_gates_let_through(B, T, H, reverse):
    """Candidates of zero: the state is c0 times the product of the gates."""
    torch, _, _ = _torch()
    p = Problem(B, T, H, "f32", reverse, seed=B + T + H)
    r = np.random.default_rng(T)
    x = 12 * r.random((B, T, H)) - 16
    x[r.random((B, T, H)) < 1 - 4 / (T + 4)] = 9.0                              # open but for a few
    p.G[:, :, :H], p.G[:, :, H:2 * H] = torch.from_numpy(x.astype(np.float32)), 0.0
    got = p.run()
    G, c0 = p.G.double().numpy(), p.c0.double().numpy()
    h, last = sr.scan_forward(G, c0, None, reverse)
    f, o, x = _sigmoid(G[:, :, :H]), _sigmoid(G[:, :, 2 * H:]), np.abs(G)
    c, E = np.abs(c0), np.zeros((B, H))
    for t in range(T - 1, -1, -1) if reverse else range(T):
        E = f[:, t] * E + (2 * x[:, t, :H] + 12) * U * f[:, t] * c
        c = f[:, t] * c
        off = np.abs(got["h"][:, t] - h[:, t])
        bound = o[:, t] * (E + (2 * x[:, t, 2 * H:] + 9) * U * c)
        assert (off <= 1.01 * bound + 2.0 ** -140).all(), (t, (off / np.maximum(bound, 1e-300)).max())
    off = np.abs(got["c_last"] - last)
    assert (off <= 1.01 * E + 2.0 ** -140).all(), (off / np.maximum(E, 1e-300)).max()
    p.check(got)
