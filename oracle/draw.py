"""Tokens drawn from rows of logits and verified drafts from their definitions, in 64 bits on the CPU (numpy).  Shares no code with the GPU path."""
from __future__ import annotations

import numpy as np

LEAST_MASS = 2.0**-40


def distribution(x, temperature):
    """softmax(x / temperature) of a row of float64 logits; None where there is none.  A temperature of 0: all on the first of the largest."""
    x = np.asarray(x, dtype=np.float64)
    if not (0 <= temperature < np.inf) or np.isnan(x).any():
        return None
    top = x.max()
    if top == -np.inf:
        return np.zeros_like(x)
    if temperature == 0:
        p = np.zeros_like(x)
        p[int(np.argmax(x))] = 1.0
        return p
    if top == np.inf:
        return None
    with np.errstate(over="ignore"):
        e = np.exp((x - top) / temperature)
    return e / e.sum()


def pick(w, u):
    """The first column whose cumulated weight is beyond u of the whole, the last with any where there is none, -1 where nothing has."""
    if not (w > 0).any():
        return -1
    sums = np.cumsum(w)
    past = np.nonzero((sums > max(u, 0.0) * sums[-1] if u == u else sums > 0) & (w > 0))[0]
    return int(past[0]) if past.size else int(np.nonzero(w > 0)[0][-1])


def margin(w, u):
    """How far u of the whole is from the nearest border between columns, as a part of the whole: how large an error of a sum changes the pick."""
    if not (w > 0).any():
        return np.inf
    sums = np.cumsum(w)
    return float(np.abs(sums[:-1] / sums[-1] - u).min()) if w.size > 1 else np.inf


def sample(x, u, temperature):
    """(token, margin) of a row."""
    p = distribution(x, temperature)
    return (-1, np.inf) if p is None else (pick(p, u), margin(p, u))


def verify(target, drafts, u, draft, temperature):
    """(tokens [G + 1], accepted, margin) of a sequence: target [G + 1, M], drafts [G], u [G + 1], draft [G, M] or None."""
    G, M = len(drafts), target.shape[1]
    tokens, near = [], np.inf
    while True:
        i = len(tokens)
        d = int(drafts[i]) if i < G else -1
        p = distribution(target[i], temperature)
        w = p
        if 0 <= d < M and p is not None:
            if draft is None or temperature == 0:
                q = np.zeros(M)
                q[d] = 1.0
            else:
                q = distribution(draft[i], temperature)
            if q is not None:
                if p[d] > 0 or q[d] > 0:
                    near = min(near, abs(u[i] * q[d] - p[d]))
                if u[i] * q[d] < p[d]:
                    tokens.append(d)
                    continue
                rest = np.maximum(p - q, 0.0)
                w = rest if rest.sum() > LEAST_MASS else p
            else:
                w = None
        break
    accepted = len(tokens)
    token = -1 if w is None else pick(w, u[G])
    near = min(near, np.inf if w is None else margin(w, u[G]))
    return tokens + [token] + [-1] * (G - accepted), accepted, near
