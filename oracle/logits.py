"""fp64 oracle of the operators on arrays of logits (numpy, row by row): test infrastructure only."""
from __future__ import annotations

import numpy as np


def lse(z, tau=1.0):
    """ln sum_v exp(z_v / tau); -inf where every z is, NaN with a NaN or +inf among them."""
    z = np.asarray(z, np.float64) / tau
    if np.isnan(z).any() or np.isposinf(z).any():
        return np.nan
    m = z.max()
    return -np.inf if np.isneginf(m) else m + np.log(np.exp(z - m).sum())


def softmax(z, tau=1.0):
    z = np.asarray(z, np.float64)
    if np.isneginf(z).all():
        return np.zeros(len(z))
    with np.errstate(invalid="ignore"):
        e = np.exp((z - z.max()) / tau)  # (not by way of lse, which swallows ln V where z is huge)
        return e / e.sum()


def top(z, K, tau=1.0):
    """(ids, vals, lse) of one row: descending, the lower id first among equals, a NaN as -inf."""
    v = np.where(np.isnan(z), -np.inf, z).astype(np.float64)
    ids = np.lexsort((np.arange(len(v)), -v))[:K]
    return ids.astype(np.int32), v[ids], lse(z, tau)


def distill(z, ids, vals, n=None, y=-1, weight=1.0, tau=1.0, alpha=1.0, scale=1.0):
    """(loss, gradient) of one row.  n: the teacher's lse at tau, or None."""
    V = len(z)
    grad = np.zeros(V)
    if weight == 0.0:
        return 0.0, grad
    there = [(int(i), float(t) / tau) for i, t in zip(ids, vals) if 0 <= i < V and not np.isneginf(t)]
    if n is None:
        n = lse([t for _, t in there]) if there else 0.0
    q, q1 = softmax(z, tau), softmax(z)
    empty = np.isneginf(np.max(z))  # (no logarithm of its softmax is asked for)
    ln_q, ln_q1 = (np.asarray(z, np.float64) / t - (0.0 if empty else lse(z, t)) for t in (tau, 1.0))
    kd = mass = 0.0
    for i, t in there:
        p = np.exp(t - n)
        mass += p
        kd += p * (t - n - (-np.inf if empty else ln_q[i]))
        grad[i] -= alpha * tau * p
    loss = alpha * tau * tau * kd if alpha > 0 else 0.0
    grad += alpha * tau * mass * q
    if alpha < 1.0 and 0 <= y < V:
        loss += (1.0 - alpha) * (np.inf if empty else -ln_q1[y])
        grad += (1.0 - alpha) * q1
        grad[y] -= 1.0 - alpha
    return weight * loss, scale * weight * grad


def draw(r, u):
    """First v whose sum of weights over words <= v exceeds u times the whole; -1 where the weights are no numbers or 0."""
    c = np.cumsum(r)
    if not np.isfinite(c[-1]) or c[-1] <= 0:
        return -1
    above = np.nonzero(c > u * c[-1])[0]
    return int(above[0]) if len(above) else int(np.nonzero(r > 0)[0][-1])


def verify(target, drafts, u, draft=None, length=None, tau=1.0, tau_draft=1.0):
    """One text: target [K+1][V], drafts [K], u [K+1], draft [K][V] or None.  Returns (accepted, tokens [K+1])."""
    V, K = target.shape[1], len(drafts)
    length = K if length is None else min(max(int(length), 0), K)
    tokens = np.full(K + 1, -1, np.int32)
    for i in range(length + 1):
        p = softmax(target[i], tau)
        if i == length:
            tokens[i] = draw(p, float(u[K]))
            return i, tokens
        d = int(drafts[i])
        q = softmax(draft[i], tau_draft) if draft is not None else (np.arange(V) == d).astype(np.float64)
        if 0 <= d < V and float(u[i]) * q[d] < p[d]:
            tokens[i] = d
            continue
        with np.errstate(invalid="ignore"):
            r = np.maximum(p - q, 0.0)
        tokens[i] = draw(p if r.sum() == 0 else r, float(u[K]))
        return i, tokens
