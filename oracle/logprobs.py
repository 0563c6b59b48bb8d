"""Log probabilities of given tokens, entropy, top alternatives and their gradient,
in fp64 numpy, one row at a time. Test infrastructure only."""
from __future__ import annotations

import numpy as np


def row(x, token, top: int):
    """(logprob, entropy, lse, [(token, logprob)] * top) of one row of logits."""
    x = np.asarray(x, dtype=np.float64)
    V = x.size
    nan = float("nan")
    if np.any(np.isnan(x)) or np.any(x == np.inf):
        return (0.0 if token < 0 else nan), nan, nan, [(-1, nan)] * top
    allowed = [v for v in range(V) if x[v] > -np.inf]
    if not allowed:
        lp = 0.0 if token < 0 else nan if token >= V else -np.inf
        return lp, 0.0, -np.inf, [(-1, -np.inf)] * top
    m = x.max()
    e = np.exp(x - m)
    log_s = np.log(e.sum())
    lse = m + log_s
    lp = 0.0 if token < 0 else nan if token >= V else (x[token] - m) - log_s
    p = e[allowed] / e.sum()
    logp = x[allowed] - m - log_s
    entropy = -float((p * logp).sum())
    order = sorted(allowed, key=lambda v: (-x[v], v))[:top]
    alts = [(v, (x[v] - m) - log_s) for v in order]
    return lp, entropy, lse, alts + [(-1, -np.inf)] * (top - len(alts))


def gradient(x, token, lse, entropy, g, h):
    """d(g logprob + h entropy) / dx of one row, with p = e^(x - lse)."""
    x = np.asarray(x, dtype=np.float64)
    V = x.size
    if np.isnan(lse) or token >= V:
        return np.full(V, np.nan)
    if lse == -np.inf:
        return np.zeros(V)
    g = g if token >= 0 else 0.0
    d = np.zeros(V)
    for v in range(V):
        if x[v] > -np.inf:
            lp = x[v] - lse
            p = np.exp(lp)
            d[v] = -g * p - h * p * (lp + entropy)
    if token >= 0:
        d[token] += g
    return d
