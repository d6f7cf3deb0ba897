"""Operators on rows of logits in float64 (oracle, test use only): a teacher's record, the distillation loss against
it with its gradient, and the class drawn with temperature, top-k, top-p and min-p.

Not from the paper: they follow their definitions, which include/snn.h states. Everything is a loop over rows, and the
drawing works on Python integers, so nothing is summed in floating point there.
"""
from __future__ import annotations

import math

import numpy as np

UNIT = 1 << 31


def log_sum_exp(x: np.ndarray) -> float:
    m = np.max(x) if x.size else -np.inf
    if np.isinf(m):
        return float(m)
    return float(m + np.log(np.sum(np.exp(x - m))))


def from_largest(x: np.ndarray) -> np.ndarray:
    """What a softmax does not see taken away: beside a type's lowest value even 64 bits keep nothing of a logarithm."""
    m = np.max(x) if x.size else -np.inf
    return x - m if np.isfinite(m) else x


def order(z: np.ndarray) -> np.ndarray:
    """Classes by logit, largest first, equal ones by class; NaN as -inf."""
    z = np.where(np.isnan(z), -np.inf, z)
    return np.lexsort((np.arange(len(z)), -z))


def top(z: np.ndarray, K: int, tau: float):
    """(ids, vals, lse) of rows z [R, C]."""
    R = len(z)
    ids, vals, lse = np.full((R, K), -1), np.full((R, K), -np.inf), np.empty(R)
    for r in range(R):
        x = np.where(np.isnan(z[r]), -np.inf, z[r].astype(np.float64))
        o = order(x)[:K]
        o = o[x[o] > -np.inf]
        ids[r, :len(o)], vals[r, :len(o)] = o, x[o]
        lse[r] = log_sum_exp(x / tau)
    return ids, vals, lse


def distill_row(z, ids, vals, lse, tau):
    """(loss, gradient, envelope, share) of one row; lse None: the entries are all of the teacher. The envelope is the
    gradient's formula with its terms in absolute value, share the student's distribution among the classes not listed."""
    C = len(z)
    z = z.astype(np.float64)
    if np.isnan(z).any() or (z == np.inf).any():
        return np.nan, np.full(C, np.nan), np.full(C, np.nan), np.zeros(C)
    of, z = z, from_largest(z) / tau
    ok = (ids >= 0) & (ids < C)
    k, v = ids[ok], vals[ok].astype(np.float64)
    v = (from_largest(v) if lse is None else v) / tau
    whole = log_sum_exp(z)
    q = np.exp(z - whole) if whole > -np.inf else np.zeros(C)
    logq = z - whole if whole > -np.inf else np.full(C, -np.inf)
    other = np.ones(C, bool)
    other[k] = False
    logq_t = log_sum_exp(logq[other]) if other.any() else -np.inf
    if lse is None:
        logp, p_t = (v - log_sum_exp(v) if len(v) and np.max(v) > -np.inf else np.full(len(v), -np.inf)), 0.0
    else:
        logp = v - float(lse)
        p_t = max(0.0, 1.0 - np.exp(logp).sum()) if other.any() else 0.0
    p = np.exp(logp)
    mass = p.sum() + p_t
    loss = sum(a * (la - lb) for a, la, lb in zip(p, logp, logq[k]) if a != 0)
    if p_t > 0:
        loss += p_t * (math.log(p_t) - logq_t)
    share = np.zeros(C)
    if logq_t > -np.inf:
        e = np.exp(from_largest(of[other]) / tau)
        share[other] = e / e.sum()
    target = p_t * share
    target[k] = p
    return loss, (mass * q - target) / tau, (mass * q + target) / tau, share


def distill(z, ids, vals, lse, tau, weight=None):
    """(loss, row_loss, grad, envelope, share) of rows z [R, C]."""
    R = len(z)
    w = np.full(R, 1.0 / R) if weight is None else weight.astype(np.float64)
    row_loss, grad, env, share = np.zeros(R), np.zeros(z.shape), np.zeros(z.shape), np.zeros(z.shape)
    for r in range(R):
        if w[r] == 0:
            continue
        row_loss[r], g, e, share[r] = distill_row(z[r], ids[r], vals[r], None if lse is None else lse[r], tau)
        grad[r], env[r] = w[r] * g, abs(w[r]) * e
    return float(sum(a * b for a, b in zip(w, row_loss) if a != 0)), row_loss, grad, env, share


def sample_row(z, e, u, top_k=0, top_p=1.0, min_p=0.0, greedy=False):
    """(class, kept) of one row of logits z whose e_j = exp((z_j - max z) / temperature) are given in float32, and the
    sum of the kept weights and the drawn one."""
    C = len(z)
    x = np.where(np.isnan(z), -np.inf, z)
    if not (x > -np.inf).any():
        return -1, 0, 0, 0
    n = [int(v) for v in np.rint(np.where(x > -np.inf, e.astype(np.float64), 0.0) * UNIT)]
    by = [int(j) for j in order(x)]
    k = C if top_k <= 0 else min(top_k, C)
    if greedy:
        k = 1
    by = [j for j in by[:k] if n[j] > 0]
    total = sum(n[j] for j in by)
    p = float(np.float32(top_p))
    limit = total if p >= 1.0 else (max(1, math.ceil(p * float(total))) if p > 0.0 else 1)
    kept, so_far = set(), 0
    least = np.float32(min(max(float(np.float32(min_p)), 0.0), 1.0)) if min_p == min_p else np.float32(0.0)
    for j in by:
        if so_far >= limit:
            break
        so_far += n[j]
        if e[j] >= least:
            kept.add(j)
    total = sum(n[j] for j in kept)
    point = min(max(math.floor(float(np.float32(u)) * float(total)) if u == u else 0, 0), total - 1)
    so_far = 0
    for j in range(C):
        if j in kept:
            so_far += n[j]
            if so_far > point:
                return j, len(kept), total, n[j]
    raise AssertionError("no class drawn")
