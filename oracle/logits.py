"""The operators on rows of logits from their definitions, in 64 bits on the CPU (numpy).  Shares no code with the GPU path.

Each function takes rows of float64 logits x [N, M] and returns float64 arrays.  Probabilities of a row of nothing but -inf are 0, its
log-sum-exp is -inf, its entropy 0."""
from __future__ import annotations

import numpy as np


def log_softmax(x, temperature=1.0):
    """(ln q [N, M], log-sum-exp [N]) of q = softmax(x / temperature)."""
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        y = np.asarray(x, dtype=np.float64) / temperature
        m = y.max(axis=1, keepdims=True)
        m = np.where(m == -np.inf, 0.0, m)
        ln_s = np.log(np.exp(y - m).sum(axis=1, keepdims=True))
        # (not y - lse: that has no digits left where all of a row is the type's lowest value)
        return np.where(ln_s == -np.inf, -np.inf, (y - m) - ln_s), (m + ln_s)[:, 0]


def entropy(logq):
    """-sum q ln q of each row."""
    with np.errstate(invalid="ignore"):
        q = np.exp(logq)
        return -np.where(q == 0, 0.0, q * logq).sum(axis=1)


def token_logprobs(x, tokens, temperature=1.0):
    """ln q at tokens [N, G], 0 for those outside the row."""
    logq, _ = log_softmax(x, temperature)
    ok = (tokens >= 0) & (tokens < x.shape[1])
    return np.where(ok, np.take_along_axis(logq, np.where(ok, tokens, 0), axis=1), 0.0)


def top(x, k):
    """Columns [N, k] of the k largest logits, largest first, equal ones by column."""
    return np.argsort(-np.asarray(x, dtype=np.float64), axis=1, kind="stable")[:, :k]


def token_gradient(x, tokens, grad, grad_entropy=None, temperature=1.0):
    """Gradient of sum_g grad_g ln q(token_g) + grad_entropy * entropy with respect to x."""
    N, M = x.shape
    logq, lse = log_softmax(x, temperature)
    q = np.exp(logq)
    out = np.zeros((N, M))
    for n in range(N):
        if lse[n] == -np.inf:
            continue
        for t, g in zip(tokens[n], grad[n]):
            if 0 <= t < M:
                out[n] -= g * q[n]
                out[n, t] += g
    if grad_entropy is not None:
        h = entropy(logq)
        out -= grad_entropy[:, None] * q * (np.where(q == 0, 0.0, logq) + h[:, None])
    return out / temperature


def teacher(vals, cols, M, temperature=1.0, log_probs=False):
    """The entries' (p, ln p, column), 0 where an entry does not count."""
    vals = np.asarray(vals, dtype=np.float64)
    ok = (cols >= 0) & (cols < M) & (vals > -np.inf)
    masked = np.where(ok, vals, -np.inf)
    lp = masked if log_probs else log_softmax(masked, temperature)[0]
    p = np.where(ok, np.exp(lp), 0.0)
    ok &= p > 0
    return np.where(ok, p, 0.0), np.where(ok, lp, 0.0), np.where(ok, cols, 0)


def distill(x, vals, cols, temperature=1.0, log_probs=False):
    """Loss of each row."""
    p, lp, at = teacher(vals, cols, x.shape[1], temperature, log_probs)
    lq = np.take_along_axis(log_softmax(x, temperature)[0], at, axis=1)
    with np.errstate(invalid="ignore"):
        return np.where(p > 0, p * (lp - lq), 0.0).sum(axis=1)


def distill_gradient(x, vals, cols, grad, temperature=1.0, log_probs=False):
    """Gradient of sum_n grad_n loss_n with respect to x."""
    N, M = x.shape
    p, _, at = teacher(vals, cols, M, temperature, log_probs)
    logq, lse = log_softmax(x, temperature)
    out = np.exp(logq) * p.sum(axis=1, keepdims=True)
    np.add.at(out, (np.arange(N)[:, None], at), -p)
    out[lse == -np.inf] = 0.0
    return out * (grad[:, None] / temperature)
