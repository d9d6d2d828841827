"""TEST INFRASTRUCTURE: log probabilities of tokens, the distance from a teacher, and their gradients, in float64 and row by row.

Nothing here is shared with the HIP path.
"""
from __future__ import annotations

import numpy as np


def _distribution(row, temperature):
    """(log probabilities, log sum) of a row of logits, or None where it has none."""
    if np.isnan(row).any() or (row == np.inf).any() or (row == -np.inf).all():
        return None
    z = row / temperature
    d = z - z.max()  # the largest may be so large that a sum with it loses the logarithm
    log = np.log(np.exp(d).sum())
    return d - log, z.max() + log


def _weighted(p, v):
    """p v, 0 where p is."""
    return np.where(p > 0, p * np.where(p > 0, v, 0.0), 0.0)


def ref_token_logprobs(logits, targets, count: int = 0, temperature: float = 1.0) -> dict:
    """logprobs, log_sums, entropies [rows] and top_logprobs, top_tokens [rows, count]; targets may be None."""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    out = dict(logprobs=np.zeros(rows), log_sums=np.zeros(rows), entropies=np.zeros(rows), top_logprobs=np.full((rows, count), -np.inf),
               top_tokens=np.full((rows, count), -1, np.int32))
    for r in range(rows):
        if targets is not None and not 0 <= targets[r] < vocab:
            continue
        d = _distribution(x[r], temperature)
        if d is None:
            for k in ("logprobs", "log_sums", "entropies"):
                out[k][r] = np.nan
            continue
        log_p, out["log_sums"][r] = d
        if targets is not None:
            out["logprobs"][r] = log_p[targets[r]]
        out["entropies"][r] = -_weighted(np.exp(log_p), log_p).sum()
        best = np.argsort(-x[r], kind="stable")[:count]
        best = best[x[r][best] > -np.inf]
        out["top_logprobs"][r, :len(best)] = log_p[best]
        out["top_tokens"][r, :len(best)] = best
    return out


def ref_token_logprobs_backward(logits, targets, log_sums, entropies, grad_logprobs, grad_entropies, temperature: float = 1.0):
    """The gradient of sum(grad_logprobs logprobs + grad_entropies entropies) by the logits, from the log sums given."""
    x = np.asarray(logits, np.float64)
    dx = np.zeros(x.shape)
    for r in range(x.shape[0]):
        g = float(grad_logprobs[r]) if targets is not None else 0.0
        h = float(grad_entropies[r]) if grad_entropies is not None else 0.0
        if (targets is not None and not 0 <= targets[r] < x.shape[1]) or (g == 0 and h == 0):
            continue
        log_p = x[r] / temperature - float(log_sums[r])
        p = np.exp(log_p)
        dx[r] = -g * p
        if grad_entropies is not None:
            dx[r] -= h * _weighted(p, log_p + float(entropies[r]))
        if targets is not None:
            dx[r, targets[r]] += g
    return dx / temperature


def ref_distill(logits, teacher, tokens, rest: bool = False, weights=None, temperature: float = 1.0) -> dict:
    """losses, log_sums, log_rests [rows], gradient [rows, vocab]; q, left: the teacher's probabilities and its rest."""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    K = teacher.shape[1]
    out = dict(losses=np.zeros(rows), log_sums=np.zeros(rows), log_rests=np.zeros(rows), gradient=np.zeros(x.shape), q=np.zeros((rows, K)),
               left=np.zeros(rows), log_p=np.zeros(x.shape))
    for r in range(rows):
        w = 1.0 if weights is None else float(weights[r])
        t, at = np.asarray(teacher[r], np.float64), np.asarray(tokens[r], np.int64)
        valid = (at >= 0) & (at < vocab) & (t != -np.inf)
        if w == 0 or not valid.any():
            continue
        t, at = t[valid], at[valid]
        d = _distribution(x[r], temperature)
        if d is None or np.isnan(t).any() or (t == np.inf).any():
            for k in ("losses", "log_sums", "gradient"):
                out[k][r] = np.nan
            if d is not None:
                out["log_sums"][r] = d[1]
            out["log_rests"][r] = np.nan if d is None and rest else 0.0
            continue
        log_p, out["log_sums"][r] = d
        log_q = t if rest else t / temperature - (np.max(t / temperature) + np.log(np.exp(t / temperature - np.max(t / temperature)).sum()))
        q = np.exp(log_q)
        named = np.zeros(vocab, bool)
        named[at] = True
        p = np.exp(log_p)
        other = p[~named].sum()
        left = max(0.0, 1.0 - q.sum()) if rest and other > 0 else 0.0
        with np.errstate(divide="ignore"):
            loss = _weighted(q, log_q - log_p[at]).sum()
            if left > 0:
                loss += left * (np.log(left) - np.log(other))
            if rest:
                out["log_rests"][r] = np.log(other) + d[1]
        dx = p * (q.sum() + left)
        np.add.at(dx, at, -q)
        if left > 0:
            dx[~named] -= left * p[~named] / other
        out["losses"][r], out["gradient"][r] = loss, dx * w / temperature
        out["q"][r, valid], out["left"][r], out["log_p"][r] = q, left, log_p
    return out
