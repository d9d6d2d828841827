"""TEST INFRASTRUCTURE: one step of a beam search and the move of the states behind it, in float64 and plain loops.

Nothing here is shared with the HIP path.
"""
from __future__ import annotations

import numpy as np


def beam_values(logits, scores, finished, pad_token: int) -> np.ndarray:
    """float64 value of every candidate [batch, beams, vocab]: score + log softmax; -inf for what is no candidate."""
    x = np.asarray(logits, np.float64)
    out = np.full(x.shape, -np.inf)
    for b in range(x.shape[0]):
        for k in range(x.shape[1]):
            s = float(scores[b, k])
            if not np.isfinite(s):
                continue
            if finished is not None and finished[b, k]:
                out[b, k, pad_token] = s
                continue
            row = x[b, k]
            if np.isnan(row).any() or (row == np.inf).any() or (row == -np.inf).all():
                continue
            d = row - row.max()
            out[b, k] = s + (d - np.log(np.exp(d).sum()))
    return out


def ref_beam_select(logits, scores, finished, pad_token: int, count: int):
    """(values float64, beams, tokens) [batch, count] of the best candidates, best first, equal ones by beam and token."""
    c = beam_values(logits, scores, finished, pad_token)
    b, K, V = c.shape
    values, parents, tokens = np.full((b, count), -np.inf), np.empty((b, count), np.int32), np.full((b, count), pad_token, np.int32)
    parents[:] = np.arange(count) % K
    for i in range(b):
        flat = c[i].reshape(-1)
        order = np.argsort(-flat, kind="stable")[:count]
        order = order[flat[order] > -np.inf]
        n = len(order)
        values[i, :n], parents[i, :n], tokens[i, :n] = flat[order], order // V, order % V
    return values, parents, tokens


def ref_beam_reorder(cache, parents) -> np.ndarray:
    """The cache [batch, beams, ...] behind the move; a parent out of range leaves its beam."""
    out = np.array(cache)
    for b in range(out.shape[0]):
        for k in range(out.shape[1]):
            p = int(parents[b, k])
            if 0 <= p < out.shape[1]:
                out[b, k] = cache[b, p]
    return out
