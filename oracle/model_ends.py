"""fp64 definitions of the operators at a model's ends: vocabulary cross
entropy, layer norm, embedding, with their gradients. Plain numpy, test
infrastructure only."""
from __future__ import annotations

import numpy as np


def logits(H, W):
    return np.asarray(H, np.float64) @ np.asarray(W, np.float64).T


def xent_forward(H, W, target, v0=0):
    """(lse, tlogit, loss) of the shard W of ids [v0, v0 + V)."""
    z = logits(H, W)
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    t = np.asarray(target) - v0
    inside = (np.asarray(target) >= 0) & (t >= 0) & (t < W.shape[0])
    tl = np.where(inside, z[np.arange(len(t)), np.where(inside, t, 0)], 0.0)
    return lse, tl, np.where(np.asarray(target) < 0, 0.0, lse - tl)


def xent_dz(H, W, target, lse, grad, v0=0):
    p = np.exp(logits(H, W) - np.asarray(lse, np.float64)[:, None])
    target = np.asarray(target)
    t = target - v0
    inside = np.flatnonzero((target >= 0) & (t >= 0) & (t < W.shape[0]))
    p[inside, t[inside]] -= 1.0
    return p * np.where(target < 0, 0.0, np.asarray(grad, np.float64))[:, None]


def xent_backward(H, W, target, lse, grad, v0=0):
    """(dH, dW): derivatives of sum(grad * loss)."""
    dz = xent_dz(H, W, target, lse, grad, v0)
    return dz @ np.asarray(W, np.float64), dz.T @ np.asarray(H, np.float64)


def norm_forward(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    var = np.square(x - mean[:, None]).mean(axis=1)
    rstd = 1.0 / np.sqrt(var + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) with the row statistics as given."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    xh = (x - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    a = dy if gamma is None else dy * gamma
    c1 = a.mean(axis=1, keepdims=True)
    c2 = (a * xh).mean(axis=1, keepdims=True)
    return np.asarray(rstd, np.float64)[:, None] * (a - c1 - xh * c2), (dy * xh).sum(axis=0), dy.sum(axis=0)


def _rows(ids, v0, V):
    r = np.asarray(ids) - v0
    return r, (r >= 0) & (r < V)


def embed_forward(ids, table, scale, v0=0):
    r, inside = _rows(ids, v0, table.shape[0])
    y = np.zeros((len(r), table.shape[1]))
    y[inside] = scale * np.asarray(table, np.float64)[r[inside]]
    return y


def embed_backward(ids, dy, V, scale, v0=0):
    r, inside = _rows(ids, v0, V)
    d = np.zeros((V, dy.shape[1]))
    np.add.at(d, r[inside], scale * np.asarray(dy, np.float64)[inside])
    return d
