"""Operators of a network on sequences of tokens in float64 (oracle, test use only): rows of an embedding and its
gradient, layer norm and its backward pass, softmax cross entropy of linear logits with both gradients, and the adjoint
of a leaky integration.

Not from the paper, except the last (the recurrence of Proposition 1): they follow their definitions, which include/snn.h
states. The bounds beside the results are the same sums with every term taken in absolute value.
"""
from __future__ import annotations

import numpy as np


def embed(E: np.ndarray, ids: np.ndarray, scale: float) -> np.ndarray:
    out = np.zeros((len(ids), E.shape[1]))
    for r, v in enumerate(ids):
        if 0 <= v < len(E):
            out[r] = scale * E[v].astype(np.float64)
    return out


def embed_grad(ids: np.ndarray, dout: np.ndarray, V: int, scale: float):
    """(dE [V, N], the same of |dout|, rows of each token)."""
    dE, bound, n = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros(V, dtype=int)
    for r, v in enumerate(ids):
        if 0 <= v < V:
            dE[v] += scale * dout[r].astype(np.float64)
            bound[v] += abs(scale) * np.abs(dout[r].astype(np.float64))
            n[v] += 1
    return dE, bound, n


def layer_norm(x, gamma, beta, eps):
    """(y, mean, rstd)."""
    x = x.astype(np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * gamma.astype(np.float64)
    return (y if beta is None else y + beta.astype(np.float64)), mean, rstd


def layer_norm_grad(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) and their bounds, at the given mean and rstd."""
    dy, k = dy.astype(np.float64), rstd.astype(np.float64)[:, None]
    h = (x.astype(np.float64) - mean.astype(np.float64)[:, None]) * k
    a = dy if gamma is None else dy * gamma.astype(np.float64)
    dx = k * (a - a.mean(1, keepdims=True) - h * (a * h).mean(1, keepdims=True))
    top = k * (np.abs(a) + np.abs(a).mean(1, keepdims=True) + np.abs(h) * np.abs(a * h).mean(1, keepdims=True))
    return (dx, (dy * h).sum(0), dy.sum(0)), (top, np.abs(dy * h).sum(0), np.abs(dy).sum(0))


def linear_ce(x, W, targets, weight=None):
    """dict of loss, row_loss, dx, dW; z_bound [R] the largest sum of |x||W| of a row, dz, p, live."""
    x, W = x.astype(np.float64), W.astype(np.float64)
    R, C = len(x), W.shape[1]
    live = (targets >= 0) & (targets < C)
    if weight is not None:
        live &= weight != 0
    n = live.sum()
    w = np.where(live, 1.0 / max(n, 1) if weight is None else np.asarray(weight, np.float64), 0.0)
    row_loss, z_bound = np.zeros(R), np.zeros(R)
    p, dz = np.zeros((R, C)), np.zeros((R, C))
    for r in np.flatnonzero(live):
        z = x[r] @ W
        z_bound[r] = np.max(np.abs(x[r]) @ np.abs(W))
        m = z.max()
        lse = m + np.log(np.exp(z - m).sum())
        row_loss[r] = lse - z[targets[r]]
        p[r] = np.exp(z - lse)
        dz[r] = w[r] * p[r]
        dz[r, targets[r]] -= w[r]
    X = np.where(live[:, None], x, 0.0)
    return dict(loss=(w * row_loss).sum(), row_loss=row_loss, dx=dz @ W.T, dW=X.T @ dz, z_bound=z_bound, dz=dz, p=p, w=w,
                live=live, X=X)


def leak_grad(x: np.ndarray, alpha: float) -> np.ndarray:
    """y [T, B, N] of x [T, B, N]."""
    y = np.zeros(x.shape)
    for t in range(len(x) - 2, -1, -1):
        y[t] = alpha * y[t + 1] + x[t + 1]
    return y
