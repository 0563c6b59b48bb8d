"""One step of beam search in fp64 numpy, one sequence at a time, and the reordering of
states. Test infrastructure only."""
from __future__ import annotations

import numpy as np


def select(x, scores, finished, pad_token: int, top: int):
    """[(total, beam, token)] * top of one sequence: x [beams, vocab], scores and finished
    [beams]."""
    x = np.asarray(x, dtype=np.float64)
    offers = []
    for b, s in enumerate(np.asarray(scores, dtype=np.float64)):
        if np.isnan(s) or s == np.inf:
            return [(np.nan, -1, -1)] * top
        if s == -np.inf:
            continue
        if finished is not None and finished[b]:
            offers.append((-s, b, 0.0, pad_token))
            continue
        if np.any(np.isnan(x[b])) or np.any(x[b] == np.inf):
            return [(np.nan, -1, -1)] * top
        m = x[b].max()
        if m == -np.inf:
            continue
        lse = np.log(np.exp(x[b] - m).sum())
        some = np.nonzero(x[b] > -np.inf)[0]
        best = some[np.lexsort((some, -x[b][some]))][:top]
        offers += [(-(s + ((x[b, v] - m) - lse)), b, -x[b, v], int(v)) for v in best]
    found = [(-t, b, v) for t, b, _, v in sorted(offers)[:top]]
    return found + [(-np.inf, -1, -1)] * (top - len(found))


def reorder(state, parents):
    """Rows of state [batch * beams, ...] by parents [batch, out_beams]; zeros for a parent
    that is none."""
    batch, out = parents.shape
    beams = state.shape[0] // batch
    r = np.zeros((batch * out, *state.shape[1:]), state.dtype)
    for i in range(batch):
        for j in range(out):
            if 0 <= parents[i, j] < beams:
                r[i * out + j] = state[i * beams + parents[i, j]]
    return r
