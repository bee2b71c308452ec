"""Operators on rows of logits in plain numpy float64, row by row.

TEST INFRASTRUCTURE: textbook definitions.  A row x[V] of logits, a scale s > 0:
log probabilities l = log softmax(s x); a logit of -inf has no weight, and a row
of nothing else has l = -inf and entropy 0.
"""
from __future__ import annotations

import numpy as np

F64 = np.float64
NINF = -np.inf


def log_probabilities(x, scale=1.0):
    """(max, log sum exp(scale (x - max)), log probabilities) of one row."""
    x = np.asarray(x, F64)
    m = np.fmax.reduce(x)      # of the logits that are no NaN; one that is makes the rest NaN
    if x.max() == NINF:
        return m, NINF, np.full_like(x, NINF)
    with np.errstate(invalid="ignore"):
        u = scale * (x - m)
        z = np.log(np.exp(u).sum())
    return m, z, u - z


def entropy(l):
    p = np.exp(l)
    return F64(np.nan) if np.isnan(p).any() else -(p[p > 0] * l[p > 0]).sum()


def top(x, l, k):
    """ids and log probabilities of the k largest logits, of equal ones the lower id first; -1, -inf where there are no more."""
    x = np.asarray(x, F64)
    ranked = np.lexsort((np.arange(len(x)), -np.where(np.isnan(x), NINF, x)))
    ranked = [j for j in ranked[:k] if x[j] > NINF]
    ids, lp = np.full(k, -1, np.int32), np.full(k, NINF)
    ids[:len(ranked)] = ranked
    lp[:len(ranked)] = l[ranked]
    return ids, lp


def logprob_bwd(x, target, d_logp, d_entropy, scale=1.0):
    """Gradient of d_logp * l[target] + d_entropy * H with respect to x."""
    m, _, l = log_probabilities(x, scale)
    p, H = np.exp(l), entropy(l)
    named = 0 <= target < len(p)
    a = d_logp if named else 0.0
    surprise = np.zeros_like(p)
    live = ~(p == 0)
    surprise[live] = p[live] * (l[live] + H)
    g = -a * p - d_entropy * surprise
    if named:
        g[target] += a
    return scale * g


def has_weight(x, of, scale=1.0):
    """Whether the tokens `of` a row weigh anything: their largest logit is above -inf and at most 745 (the logarithm of the least
    number of 64 bits) below the row's, times the scale."""
    x = np.asarray(x, F64)
    m = np.fmax.reduce(x[of], initial=NINF)
    return m > NINF and not scale * (m - np.fmax.reduce(x)) < -745


def distill(x, ids, t, scale=1.0, tail=False):
    """(loss, its gradient with respect to x) of one row against listed tokens and the teacher's log probabilities of them."""
    V = len(x)
    t = np.asarray(t, F64)
    there = [(int(i), F64(v)) for i, v in zip(ids, t) if 0 <= i < V and not v == NINF]
    if not there:
        return 0.0, np.zeros(V)
    _, _, l = log_probabilities(x, scale)
    p = np.exp(l)
    log_q = np.array([v for _, v in there])
    if not tail:
        n = log_q.max()
        log_q = log_q - (n + np.log(np.exp(log_q - n).sum()))
    q = np.exp(log_q)
    loss = 0.0
    for (i, _), qk, lq in zip(there, q, log_q):
        if not qk == 0:
            loss += qk * (lq - l[i])
    listed = np.zeros(V, bool)
    listed[[i for i, _ in there]] = True
    Q, rest = q.sum(), 0.0
    if tail and has_weight(x, ~listed, scale):
        rest = max(0.0, 1.0 - Q)
    if rest > 0:
        # log p of the class as a whole: p itself has few bits left, or none, where the student gives it next to nothing
        n = np.fmax.reduce(l[~listed])
        log_p_rest = n + np.log(np.exp(l[~listed] - n).sum())
        loss += rest * (np.log(rest) - log_p_rest)
    g = (Q + rest) * p
    if rest > 0:
        g[~listed] -= rest * np.exp(l[~listed] - log_p_rest)
    for (i, _), qk in zip(there, q):
        g[i] -= qk
    return loss, scale * g
