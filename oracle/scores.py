"""Plain fp64 oracle of the vocabulary row operators: token scores and
distillation from a teacher's top logits, with their gradients.

TEST INFRASTRUCTURE ONLY (same rule as ``oracle.moe``).

Each function takes one row.  ``scores`` counts a NaN logit as -infinity;
``distill`` lets it show.  Gradients are of ``g * logp + g_entropy * entropy`` and of
``g * loss`` with respect to the logits.
"""
from __future__ import annotations

import numpy as np

NAN = float("nan")


def log_softmax(l, tau=1.0):
    d = (l - np.max(l)) / tau
    return d - np.log(np.sum(np.exp(d)))


def scores(l, tau, token, m, g=0.0, g_entropy=0.0):
    """(logp, entropy, top ids, top log probabilities, gradient) of one row."""
    l = np.asarray(l, np.float64)
    l = np.where(np.isnan(l), -np.inf, l)
    V = l.size
    top = np.argsort(-l, kind="stable")[:m]
    zero = g_entropy == 0 and (g == 0 or token < 0)
    if not np.isfinite(np.max(l)):
        bad = np.full(V, 0.0 if zero else NAN)
        return (0.0 if token < 0 else NAN), NAN, top, np.full(m, NAN), bad
    lp = log_softmax(l, tau)
    p = np.exp(lp)
    h = -np.sum(p[p > 0] * lp[p > 0])
    logp = 0.0 if token < 0 else NAN if token >= V else lp[token]
    grad = np.zeros(V)
    if not zero:
        plp = np.zeros(V)
        plp[p > 0] = p[p > 0] * lp[p > 0]
        grad -= g_entropy * (plp + p * h)
        if token >= V and g != 0:
            grad[:] = NAN
        elif token >= 0:
            grad -= g * p
            grad[token] += g
    return logp, h, top, lp[top], grad / tau


def entries(ids, V):
    """The slots of a list that hold an entry: ids in [0, V), each id's first slot."""
    seen, slots = set(), []
    for j, i in enumerate(ids):
        if 0 <= i < V and i not in seen:
            seen.add(i)
            slots.append(j)
    return slots


def distill(l, ids, values, tail, tau, g=1.0):
    """(loss, gradient) of one row."""
    l = np.asarray(l, np.float64)
    V = l.size
    slots = entries(ids, V)
    if not slots:
        return 0.0, np.zeros(V)
    s = np.asarray([ids[j] for j in slots])
    v = np.asarray([values[j] for j in slots], np.float64)
    with np.errstate(all="ignore"):
        if np.isnan(l).any() or not np.isfinite(np.max(l)) or np.isnan(v).any() \
                or np.max(v) == np.inf or (not tail and np.max(v) == -np.inf):
            return NAN, np.zeros(V) if g == 0 else np.full(V, NAN)
        lq = log_softmax(l, tau)
        q = np.exp(lq)
        lp = v if tail else log_softmax(v, tau)
        p = np.exp(lp)
        on = p > 0
        loss = np.sum(p[on] * (lp[on] - lq[s][on]))
        rest = np.ones(V, bool)
        rest[s] = False
        ratio, weight = 0.0, np.sum(p) if tail else 1.0  # weight: of log sum exp(l / tau) in the loss
        if tail and np.any(l[rest] > -np.inf):
            big = max(0.0, 1.0 - np.sum(p))
            r = l[rest]
            d = (r - np.max(r)) / tau
            log_mass = (np.max(r) - np.max(l)) / tau + np.log(np.sum(np.exp(d)))
            log_mass -= np.log(np.sum(np.exp((l - np.max(l)) / tau)))
            if big > 0:
                loss += big * (np.log(big) - log_mass)
                # q_v P / Q without Q's underflow
                ratio = np.zeros(V)
                ratio[rest] = big * np.exp(d) / np.sum(np.exp(d))
                weight += big
    grad = weight * q - ratio
    grad[s] = weight * q[s] - p
    return tau * tau * loss, (g * tau * grad if g != 0 else np.zeros(V))
