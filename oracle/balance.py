"""A router's balance loss and its gradient from their definitions, in 64 bits on the CPU (numpy).  Shares no code with the GPU path."""
from __future__ import annotations

import numpy as np


def _softmax(x):
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        m = x.max(axis=1, keepdims=True)
        m = np.where(m == -np.inf, 0.0, m)
        e = np.exp(x - m)
        s = e.sum(axis=1, keepdims=True)
        return np.where(s == 0, 0.0, e / s), (m + np.log(s))[:, 0]


def loss(x, cols, groups=1):
    """(loss, z, probs, counts, rows) by groups; x [N, E], cols [N, k]."""
    N, E = x.shape
    per = N // groups
    out = [np.zeros(groups), np.zeros(groups), np.zeros((groups, E)), np.zeros((groups, E), dtype=np.int64), np.zeros(groups, dtype=np.int64)]
    real = (cols >= 0) & (cols < E)
    for g in range(groups):
        part = slice(g * per, (g + 1) * per)
        keep = real[part].any(axis=1)
        counts = np.bincount(cols[part][real[part]].astype(np.int64), minlength=E)
        n = int(keep.sum())
        out[3][g], out[4][g] = counts, n
        if n == 0:
            continue
        p, lse = _softmax(np.asarray(x[part][keep], dtype=np.float64))
        with np.errstate(invalid="ignore"):
            out[2][g] = p.sum(axis=0) / n
            out[1][g] = np.where(lse == -np.inf, 0.0, lse * lse).sum() / n
            mean = out[2][g]
            out[0][g] = E * (counts[counts > 0] * mean[counts > 0]).sum() / counts.sum()
    return out


def gradient(x, cols, counts, rows, grad_loss, grad_z=None, grad_vals=None):
    """Gradient of sum_g (grad_loss loss + grad_z z) + sum grad_vals x[picked] with respect to x; counts [groups, E], rows [groups]."""
    N, E = x.shape
    groups = counts.shape[0]
    per = N // groups
    real = (cols >= 0) & (cols < E)
    keep = real.any(axis=1)
    p, lse = _softmax(np.asarray(x, dtype=np.float64))
    out = np.zeros((N, E))
    for n in range(N):
        g = n // per
        if not keep[n]:
            continue
        over, all_picks = 1.0 / max(1, rows[g]), max(1, counts[g].sum())
        w = E * grad_loss[g] * counts[g] / all_picks * over
        out[n] = p[n] * (w - (p[n] * w).sum())
        if grad_z is not None and lse[n] != -np.inf:
            out[n] += 2 * grad_z[g] * lse[n] * over * p[n]
        if grad_vals is not None:
            for j in np.nonzero(real[n])[0]:
                out[n, cols[n, j]] += grad_vals[n, j]
    return out
