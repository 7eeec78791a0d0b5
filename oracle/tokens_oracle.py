"""CPU oracle for the operators over tokens and a vocabulary -- TEST INFRASTRUCTURE ONLY.

Embedding lookup with its gradient, layer norm with its backprop, and softmax cross entropy of a linear layer with the gradients of
both operands, from their definitions in fp64 with numpy:

    embedding            y[t] = scale * table[id[t]], 0 for ids outside the table
    embedding_bwd        dtable[v] = scale * sum over t with id[t] = v of dy[t]
    layer_norm           mean = sum x / cols, rstd = (sum (x - mean)^2 / cols + eps)^(-1/2), y = (x - mean) rstd gamma + beta
    layer_norm_bwd       of the affine map and the normalisation, from the statistics handed over
    linear_xent          z = x w^T, lse = log sum exp z, loss = lse - z[label], 0 for labels outside the vocabulary
    linear_xent_bwd      g = (exp(z - lse) - onehot) dloss, dx = g w, dw = g^T x

Pins (tests/test_oracle_pins_tokens.py): closed forms, the dense one-hot products, and central differences of every gradient.
"""
from __future__ import annotations

import numpy as np


def _f64(a):
    return np.asarray(a, dtype=np.float64)


def embedding(table, ids, scale=1.0):
    table, ids = _f64(table), np.asarray(ids)
    y = np.zeros((ids.size, table.shape[1]))
    live = (ids >= 0) & (ids < table.shape[0])
    y[live] = scale * table[ids[live]]
    return y


def embedding_bwd(dy, ids, vocab, scale=1.0):
    dy, ids = _f64(dy), np.asarray(ids)
    out = np.zeros((vocab, dy.shape[1]))
    live = (ids >= 0) & (ids < vocab)
    np.add.at(out, ids[live], dy[live])
    return scale * out


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    """-> y, mean, rstd"""
    x = _f64(x)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * _f64(gamma)
    if beta is not None:
        y = y + _f64(beta)
    return y, mean, rstd


def layer_norm_bwd(x, gamma, mean, rstd, dy):
    """-> dx, dgamma, dbeta"""
    x, dy, mean, rstd = _f64(x), _f64(dy), _f64(mean)[:, None], _f64(rstd)[:, None]
    xh = (x - mean) * rstd
    g = dy if gamma is None else dy * _f64(gamma)
    dx = rstd * (g - g.mean(axis=1, keepdims=True) - xh * (g * xh).mean(axis=1, keepdims=True))
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


def linear_xent(x, w, labels):
    """-> loss, lse"""
    z = _f64(x) @ _f64(w).T
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    labels = np.asarray(labels)
    live = (labels >= 0) & (labels < z.shape[1])
    loss = np.zeros(z.shape[0])
    loss[live] = (lse - z[np.arange(z.shape[0]), np.where(live, labels, 0)])[live]
    return loss, lse


def linear_xent_bwd(x, w, labels, lse, dloss):
    """-> dx, dw"""
    x, w, labels = _f64(x), _f64(w), np.asarray(labels)
    g = np.exp(x @ w.T - _f64(lse)[:, None])
    live = (labels >= 0) & (labels < w.shape[0])
    g[np.flatnonzero(live), labels[live]] -= 1.0
    g *= np.where(live, _f64(dloss), 0.0)[:, None]
    g[~live] = 0.0
    return g @ w, g.T @ x
