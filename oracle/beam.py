"""A step of beam search and the states that follow it, in 64 bits."""
from __future__ import annotations

import numpy as np


def candidates(logits, scores, finished=None, pad: int = 0):
    """The scores of every (beam, token) of one batch entry: logits [beams, vocab], scores [beams]."""
    x = np.asarray(logits, dtype=np.float64)
    c = np.full(x.shape, -np.inf)
    for i, row in enumerate(x):
        if not np.isfinite(scores[i]):
            continue
        if finished is not None and finished[i]:
            c[i, pad] = scores[i]
        elif not np.isnan(row).any() and not np.isposinf(row).any() and not np.isneginf(row).all():
            d = row - row.max()
            with np.errstate(divide="ignore"):
                c[i] = scores[i] + d - np.log(np.exp(d).sum())
    return c


def select(logits, scores, k: int, finished=None, pad: int = 0):
    """(scores float64, parents, tokens) [batch, k] of the best candidates, equal ones by beam and token."""
    out = []
    for b in range(len(logits)):
        c = candidates(logits[b], np.asarray(scores[b], dtype=np.float64), None if finished is None else finished[b], pad)
        # Logits of a beam that differ by less than their scores have digits are in order all the same.
        x = np.where(np.isneginf(c), 0.0, np.asarray(logits[b], dtype=np.float64))
        beam, token = np.indices(c.shape)
        at = np.lexsort([a.reshape(-1) for a in (token, -x, beam, -c)])[:k]
        out.append((c.reshape(-1)[at], at // c.shape[1], at % c.shape[1]))
    return tuple(np.stack(t) for t in zip(*out))


def reorder(x, parents):
    """y[b, j] = x[b, parents[b, j]]."""
    x = np.asarray(x)
    return np.stack([x[b, np.asarray(p)] for b, p in enumerate(parents)])
