"""fp64 oracle of the operators that adapt a trained model: from the definitions, row by row, in numpy."""
from __future__ import annotations

import numpy as np


def softmax(z, tau=1.0):
    with np.errstate(invalid="ignore"):
        t = np.asarray(z, np.float64) / tau
        e = np.exp(t - t.max())
    return e / e.sum()


def word_logp(z, y, tau=1.0):
    t = np.asarray(z, np.float64) / tau
    if t[y] == -np.inf:
        return -np.inf
    m = t.max()
    return t[y] - m - np.log(np.exp(t - m).sum())


def _gradient(z, y, g, tau):
    """g ([v = y] - softmax(z / tau)) / tau"""
    d = -softmax(z, tau) * g
    d[y] += g
    return d / tau


def policy(z, y, advantage, old=None, ref=None, weight=None, tau=1.0, lo=0.2, hi=0.2, beta=0.0, scale=1.0):
    """(loss, logp, dlogits, g): g the derivatives of the unweighted losses with respect to the log-probabilities."""
    rows, V = z.shape
    loss, logp, dz, gs = np.zeros(rows), np.zeros(rows), np.zeros((rows, V)), np.zeros(rows)
    for m in range(rows):
        w = 1.0 if weight is None else float(weight[m])
        if not 0 <= y[m] < V or w == 0.0:
            continue
        l, A = word_logp(z[m], y[m], tau), float(advantage[m])
        rho = 1.0 if old is None else np.exp(l - float(old[m]))
        held = min(max(rho, 1.0 - lo), 1.0 + hi)
        loss[m] = -min(rho * A, held * A)
        g = 0.0 if rho * A > held * A else -rho * A
        if beta:
            d = float(ref[m]) - l
            loss[m] += beta * (np.expm1(d) - d if d < np.inf else np.inf)
            g -= beta * np.expm1(d)
        loss[m] *= w
        logp[m] = l
        if l > -np.inf:
            gs[m] = g
            dz[m] = _gradient(z[m], y[m], g * w * scale, tau)
    return loss, logp, dz, gs


def preference(z, y, ref=None, weight=None, kind="logistic", beta=0.1, smoothing=0.0, mean=False, scale=1.0):
    """z [T][2 P][V].  (loss [P], S [2 P], dlogits, r [P], derivatives of the unweighted losses by r)."""
    T, B, V = z.shape
    P = B // 2
    w = np.ones(P) if weight is None else np.asarray(weight, np.float64)
    counts = (y >= 0) & (y < V) & (np.concatenate([w, w]) != 0.0)
    l = np.array([[word_logp(z[t, s], y[t, s]) if counts[t, s] else 0.0 for s in range(B)] for t in range(T)]).reshape(T, B)
    n = np.maximum(counts.sum(0), 1) if mean else np.ones(B)
    S = l.sum(0) / n
    against = S if ref is None else S - np.asarray(ref, np.float64)
    with np.errstate(invalid="ignore"):
        r = against[:P] - against[P:]
    if kind == "logistic":
        with np.errstate(invalid="ignore"):
            up, down = np.logaddexp(0.0, -beta * r), np.logaddexp(0.0, beta * r)
        loss = (1.0 - smoothing) * up + (smoothing * down if smoothing else 0.0)
        g = beta * (smoothing * np.exp(-up) - (1.0 - smoothing) * np.exp(-down))
    elif kind == "squared":
        loss, g = (r - 0.5 / beta) ** 2, 2.0 * (r - 0.5 / beta)
    else:
        loss, g = np.maximum(0.0, 1.0 - beta * r), np.where(beta * r >= 1.0, 0.0, np.where(np.isnan(r), np.nan, -beta))
    dz = np.zeros((T, B, V))
    for t in range(T):
        for s in range(B):
            if counts[t, s] and l[t, s] > -np.inf:
                f = g[s % P] * w[s % P] * scale / n[s] * (1.0 if s < P else -1.0)
                dz[t, s] = _gradient(z[t, s], y[t, s], f, 1.0)
    return np.where(w == 0.0, 0.0, w * np.where(w == 0.0, 0.0, loss)), S, dz, r, g


def adapter_forward(x, down, up, ids, scale=None, base=None):
    """x [M][K], down [n][R][K], up [n][N][R], ids [M] (outside [0, n): none).  (out [M][N], inner [M][R])."""
    M, n, R, N = len(x), len(down), down.shape[1], up.shape[1]
    out = np.zeros((M, N)) if base is None else np.array(base, np.float64)
    inner = np.zeros((M, R))
    for m in range(M):
        if 0 <= ids[m] < n:
            inner[m] = down[ids[m]] @ x[m]
            out[m] += (1.0 if scale is None else float(scale[ids[m]])) * (up[ids[m]] @ inner[m])
    return out, inner


def adapter_backward(dout, x, inner, down, up, ids, scale=None):
    """(ddown, dup, dx) of sum(dout * out)."""
    M, n = len(x), len(down)
    ddown, dup, dx = np.zeros(down.shape), np.zeros(up.shape), np.zeros(x.shape)
    for m in range(M):
        a = ids[m]
        if 0 <= a < n:
            f = 1.0 if scale is None else float(scale[a])
            dinner = f * (up[a].T @ dout[m])
            dup[a] += f * np.outer(dout[m], inner[m])
            ddown[a] += np.outer(dinner, x[m])
            dx[m] = down[a].T @ dinner
    return ddown, dup, dx
