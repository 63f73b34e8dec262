"""float64 definitions of the vocabulary's operators (include/echovocab.h) and of gradient clipping (include/echoclip.h)."""
from __future__ import annotations

import numpy as np


def embed_forward(tokens, table, scale):
    table = np.asarray(table, np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for n, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[n] = scale * table[t]
    return out


def embed_backward(tokens, dout, scale, V):
    """dtable, and the sum of the magnitudes added into each entry."""
    dout = np.asarray(dout, np.float64)
    dtable, size = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1]))
    word = (np.asarray(tokens) >= 0) & (np.asarray(tokens) < V)
    np.add.at(dtable, np.asarray(tokens)[word], scale * dout[word])
    np.add.at(size, np.asarray(tokens)[word], abs(scale) * np.abs(dout[word]))
    return dtable, size


def labelled(labels, V):
    labels = np.asarray(labels)
    return np.flatnonzero((labels >= 0) & (labels < V))


def loss_forward(h, W, labels, eps):
    """loss [N], lse [N]; zeros for rows without a label."""
    h, W, labels = np.asarray(h, np.float64), np.asarray(W, np.float64), np.asarray(labels)
    loss, lse = np.zeros(len(h)), np.zeros(len(h))
    rows = labelled(labels, len(W))
    if len(rows) == 0:
        return loss, lse
    z = h[rows] @ W.T
    top = z.max(1, keepdims=True)
    lse[rows] = top[:, 0] + np.log(np.exp(z - top).sum(1))
    loss[rows] = lse[rows] - (1 - eps) * z[np.arange(len(rows)), labels[rows]] - eps * z.mean(1)
    return loss, lse


def loss_backward(dloss, h, W, labels, eps):
    """dh [N,D], dW [V,D] and dz of the rows with a label."""
    h, W, labels = np.asarray(h, np.float64), np.asarray(W, np.float64), np.asarray(labels)
    dh, dW = np.zeros_like(h), np.zeros_like(W)
    rows = labelled(labels, len(W))
    if len(rows) == 0:
        return dh, dW, np.zeros((0, len(W)))
    z = h[rows] @ W.T
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    dz = p - eps / len(W)
    dz[np.arange(len(rows)), labels[rows]] -= 1 - eps
    dz *= np.asarray(dloss, np.float64)[rows, None]
    dh[rows] = dz @ W
    dW[:] = dz.T @ h[rows]
    return dh, dW, dz


def grad_norm(grads):
    return float(np.sqrt(sum((np.asarray(g, np.float64) ** 2).sum() for g in grads)))


def grad_clip(grads, max_norm):
    norm = grad_norm(grads)
    f = max_norm / norm if max_norm < norm < 2.0 ** 128 - 2.0 ** 103 else 1.0      # from there on fp32 rounds a norm to infinity
    return norm, [np.asarray(g, np.float64) * f for g in grads]
