"""float64 definitions of the gated linear recurrence (include/echoscan.h), the distillation (include/echodistill.h) and the verification of
drafted words (include/echodraft.h)."""
from __future__ import annotations

import numpy as np


def _sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def lengths(n, B, T):
    return np.full(B, T) if n is None else np.clip(np.asarray(n, np.int64), 0, T)


def _order(n, reverse):
    return range(n - 1, -1, -1) if reverse else range(n)


def scan_forward(G, c0, n, reverse=False):
    """h [B,T,H], c_last [B,H]"""
    G = np.asarray(G, np.float64)
    B, T, H3 = G.shape
    H = H3 // 3
    h, last = np.zeros((B, T, H)), np.zeros((B, H)) if c0 is None else np.array(c0, np.float64)
    for b, m in enumerate(lengths(n, B, T)):
        for t in _order(m, reverse):
            f, g, o = _sigmoid(G[b, t, :H]), np.tanh(G[b, t, H:2 * H]), _sigmoid(G[b, t, 2 * H:])
            last[b] = f * last[b] + _sigmoid(-G[b, t, :H]) * g
            h[b, t] = o * last[b]
    return h, last


def scan_backward(dh, dc_last, G, c0, n, reverse=False):
    """dG [B,T,3H], dc0 [B,H]"""
    G, dh = np.asarray(G, np.float64), np.asarray(dh, np.float64)
    B, T, H3 = G.shape
    H = H3 // 3
    dG, dc0 = np.zeros((B, T, H3)), np.zeros((B, H)) if dc_last is None else np.array(dc_last, np.float64)
    for b, m in enumerate(lengths(n, B, T)):
        c = np.zeros(H) if c0 is None else np.asarray(c0[b], np.float64)
        before = {}
        for t in _order(m, reverse):
            before[t] = c
            c = _sigmoid(G[b, t, :H]) * c + _sigmoid(-G[b, t, :H]) * np.tanh(G[b, t, H:2 * H])
        for t in reversed(list(_order(m, reverse))):
            f, k, g, o = _sigmoid(G[b, t, :H]), _sigmoid(-G[b, t, :H]), np.tanh(G[b, t, H:2 * H]), _sigmoid(G[b, t, 2 * H:])
            c = f * before[t] + k * g
            r = dh[b, t] * o + dc0[b]
            dG[b, t] = np.concatenate([r * (before[t] - g) * f * k, r * k * (1 - g * g), dh[b, t] * c * o * _sigmoid(-G[b, t, 2 * H:])])
            dc0[b] = f * r
    return dG, dc0


def teacher_rows(words, logits, V, T):
    """For each row that has entries: (row, words, shares, log shares)"""
    for n, (w, t) in enumerate(zip(np.asarray(words), np.asarray(logits, np.float64))):
        in_ = (w >= 0) & (w < V) & (t != -np.inf)
        if in_.any():
            x = t[in_] / T
            x = x - x.max()
            log_q = x - np.log(np.exp(x).sum())
            yield n, w[in_], np.exp(log_q), log_q


def distill_forward(h, W, words, logits, T):
    """loss [N], lse [N]; zeros for rows without entries"""
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    loss, lse = np.zeros(len(h)), np.zeros(len(h))
    for n, w, q, log_q in teacher_rows(words, logits, len(W), T):
        z = W @ h[n] / T
        lse[n] = z.max() + np.log(np.exp(z - z.max()).sum())
        loss[n] = T * T * (q * (log_q - z[w] + lse[n])).sum()
    return loss, lse


def distill_backward(dloss, h, W, words, logits, T):
    """dh [N,D], dW [V,D], and dz [N,V]"""
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    dz = np.zeros((len(h), len(W)))
    for n, w, q, _ in teacher_rows(words, logits, len(W), T):
        z = W @ h[n] / T
        p = np.exp(z - z.max())
        dz[n] = p / p.sum()
        np.subtract.at(dz[n], w, q)
        dz[n] *= T * float(dloss[n])
    rows = sorted(n for n, *_ in teacher_rows(words, logits, len(W), T))
    dW = dz[rows].T @ h[rows] if rows else np.zeros_like(W)
    return dz @ W, dW, dz


def draft_verify(drafted, n_drafted, draft, target, u, r):
    """tokens [B,K+1], taken [B]"""
    target, draft = np.asarray(target, np.float64), np.asarray(draft, np.float64)
    B, K, V = draft.shape
    tokens, taken = np.full((B, K + 1), -1, np.int64), np.zeros(B, np.int64)

    def usable(w):
        return np.where((w > 0) & (w < np.inf), w, 0.0)          # NaN compares false

    with np.errstate(invalid="ignore"):
        for b, n in enumerate(lengths(n_drafted, B, K)):
            a = 0
            while a < n and 0 <= drafted[b][a] < V and float(u[b][a]) * draft[b, a, drafted[b][a]] < target[b, a, drafted[b][a]]:
                tokens[b, a] = drafted[b][a]
                a += 1
            taken[b] = a
            w = usable(target[b, a] - draft[b, a]) if a < n else usable(target[b, a])
            if not w.any():
                w = usable(target[b, a])
            if w.any():
                sums = np.cumsum(w)
                x = float(r[b])
                pass_ = np.flatnonzero(sums > (x if x > 0 else 0.0) * sums[-1])
                tokens[b, a] = pass_[0] if len(pass_) else np.flatnonzero(w)[-1]
    return tokens, taken
