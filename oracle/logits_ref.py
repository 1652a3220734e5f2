"""The operators on logits, from their definitions, in 64 bits, one row at a time (numpy).

A row's order: value descending, index ascending; -inf (and, for sampling and the top logits, NaN) is not in it.  A weight is
exp((z - max z) / T); with an infinite maximum the infinite logits have weight 1 and the others 0.
"""
import math

import numpy as np


def order_of(z):
    """Indexes of the row's order."""
    z = np.asarray(z, dtype=np.float64)
    there = np.flatnonzero(~np.isnan(z) & (z != -np.inf))
    return there[np.argsort(-z[there], kind="stable")]


def weights(z, T):
    z = np.asarray(z, dtype=np.float64)
    some = z[~np.isnan(z)]
    best = some.max() if len(some) else -np.inf
    if best == -np.inf:
        return np.zeros(len(z))
    if best == np.inf:
        return (z == np.inf).astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        t = (z - best) / T
    return np.where(np.isnan(t) | (z == -np.inf), 0.0, np.exp(np.where(np.isnan(t), 0.0, t)))


def sample_row(z, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(class, ln of its probability among the candidates)."""
    order = order_of(z)
    if len(order) == 0:
        return -1, -math.inf
    if not T > 0:
        return int(order[0]), 0.0
    w = weights(z, T)
    sorted_w = w[order]
    keep = np.ones(len(order), dtype=bool)
    if top_k > 0:
        keep &= np.arange(len(order)) < top_k
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(sorted_w)[:-1]])
        keep &= before < top_p * sorted_w.sum()
        keep[0] = True
    if min_p > 0:
        keep &= sorted_w >= min(min_p, 1.0)
    members = np.sort(order[keep])
    upto = np.cumsum(w[members])
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0  # (the largest float32 below 1)
    j = int(members[np.searchsorted(upto, u * upto[-1], side="right")])
    return j, math.log(w[j] / upto[-1])


def top_row(z, k, T=1.0):
    """(values [k], classes [k], probability of the others)."""
    z = np.asarray(z, dtype=np.float64)
    order = order_of(z)[:k]
    values, classes = np.full(k, -np.inf), np.full(k, -1, dtype=np.int64)
    values[:len(order)], classes[:len(order)] = z[order], order
    w = weights(z, T)
    total = w.sum()
    others = np.ones(len(z), dtype=bool)
    others[order] = False
    return values, classes, w[others].sum() / total if total > 0 else 0.0


def list_of(classes, n):
    """Positions of the entries that count: the class exists and stands in no earlier entry."""
    seen, out = set(), []
    for i, c in enumerate(classes):
        if 0 <= c < n and c not in seen:
            seen.add(c)
            out.append(i)
    return out


def distill_row(z, values, classes, rest=0.0, T=1.0):
    """(loss, gradient by z, for each class the sum of the magnitudes that the gradient is the difference of).  A loss beyond the
    range of float32 is infinite, as in the operator's output."""
    z = np.asarray(z, dtype=np.float64)
    n = len(z)
    at = list_of(classes, n)
    c, t = np.asarray(classes)[at].astype(np.int64), np.asarray(values, dtype=np.float64)[at]
    rest = min(max(rest, 0.0), 1.0) if rest == rest else rest
    if np.isnan(z).any() or np.isnan(t).any() or rest != rest:
        return math.nan, np.full(n, math.nan), np.full(n, math.nan)
    if len(at) == 0 or t.max() == -np.inf or z.max() == -np.inf:
        return 0.0, np.zeros(n), np.zeros(n)
    e = weights(z, T)
    total = e.sum()
    others = np.ones(n, dtype=bool)
    others[c] = False
    # the mass outside the list by its own largest weight: relative to the row's largest it may be below 2^-1074
    share, log_others = np.zeros(n), -math.inf  # of each class in the others' weight; ln of that weight
    if others.any() and z[others].max() > -np.inf and (z.max() < np.inf or z[others].max() == np.inf):
        e_others = weights(z[others], T)
        share[others] = e_others / e_others.sum()
        log_others = math.log(e_others.sum()) + ((z[others].max() - z.max()) / T if z.max() < np.inf else 0.0)
    p = weights(t, T)
    p = p / p.sum() * (1.0 - rest)
    # ln q from the differences, which do not underflow
    with np.errstate(divide="ignore", invalid="ignore"):
        log_q = (z[c] - z.max()) / T - math.log(total) if z.max() < np.inf else np.log(e[c] / total)
        loss = float(np.sum(np.where(p > 0, p * (np.log(np.where(p > 0, p, 1.0)) - log_q), 0.0)))
        if rest > 0:
            loss += rest * (math.log(rest) - (log_others - math.log(total)))
    if loss >= 3.4028235677973366e38:  # (half a step above the largest float32)
        loss = math.inf
    grad = (e / total - rest * share) / T
    size = (e / total + rest * share) / T
    grad[c] = (e[c] / total - p) / T
    size[c] = (e[c] / total + p) / T
    return loss, grad, size
