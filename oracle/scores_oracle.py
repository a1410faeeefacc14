"""Oracle of the operators on rows of class scores, in float64 numpy: a
teacher's top scores, distillation from them, and labels drawn from a row's
distribution.  Plain per-row definitions; no code in common with the library.

The order of a row's classes is by falling score, the lower class first among
equals; a score of -inf takes a class out of the row.
"""
from __future__ import annotations

import numpy as np


def order(z):
    """Classes of a row in order, those of score -inf and NaN left out."""
    z = np.asarray(z, np.float64)
    c = np.flatnonzero(z > -np.inf)
    return c[np.lexsort((c, -z[c]))]


def top_logits(z, K):
    """(values, classes) of the first K classes of every row, n x K."""
    n = z.shape[0]
    vals = np.full((n, K), -np.inf)
    cls = np.full((n, K), -1, np.int32)
    for i in range(n):
        o = order(z[i])[:K]
        vals[i, :len(o)] = z[i, o]
        cls[i, :len(o)] = o
    return vals, cls


def _log_softmax(x):
    x = x - x.max()
    return x - np.log(np.exp(x).sum())


def distill(z, top_values, top_classes, T, weight=1.0, scale=1.0, mask=None, n_mask=None, base=None):
    """(loss, gradient, column sums of the gradient)."""
    n, C = z.shape
    if n_mask is None:
        n_mask = n if mask is None else int(np.count_nonzero(mask))
    grad = np.zeros((n, C)) if base is None else np.array(base, np.float64)
    loss = 0.0
    for i in range(n):
        if mask is not None and not mask[i]:
            continue
        here = (top_classes[i] >= 0) & (top_classes[i] < C) & ~(top_values[i] == -np.inf)
        if not here.any():
            continue
        cls = top_classes[i][here]
        lnq = _log_softmax(top_values[i][here].astype(np.float64) / T)
        lnp = _log_softmax(z[i].astype(np.float64) / T)
        q = np.exp(lnq)
        pos = q > 0
        loss += (q[pos] * (lnq[pos] - lnp[cls[pos]])).sum()
        g = np.exp(lnp)
        for c, w in zip(cls, q):
            g[c] -= w
        grad[i] += scale * weight * T / n_mask * g
    return weight * T * T / n_mask * loss, grad, grad.sum(0)


def sample_row(z, u, T, top_k=0, top_p=1.0, min_p=0.0):
    """(label, probability, kept classes) of one row."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or np.isposinf(z).any() or (T != 0 and not 0 <= u < 1):
        return -1, 0.0, np.zeros(0, np.int64)
    o = order(z)
    if len(o) == 0:
        return -1, 0.0, o
    if T == 0:
        return int(o[0]), 1.0, o[:1]
    x = (z[o] - z[o[0]]) / T
    m = len(o) if top_k == 0 else min(top_k, len(o))
    w = np.exp(x[:m])
    run = np.cumsum(w)
    if top_p < 1:
        m = min(m, int(np.count_nonzero(run - w < top_p * run[-1])))
    if min_p > 0:
        m = min(m, int(np.count_nonzero(x >= np.log(min_p))))
    kept = np.sort(o[:m])
    w = np.exp((z[kept] - z[o[0]]) / T)
    run = np.cumsum(w)
    k = int(np.count_nonzero(run <= u * run[-1]))
    return int(kept[k]), float(w[k] / run[-1]), kept


def sample_labels(z, u, T, top_k=0, top_p=1.0, min_p=0.0, mask=None, labels=None, prob=None):
    n = z.shape[0]
    labels = np.full(n, -7, np.int32) if labels is None else labels.copy()
    prob = np.full(n, -7.0) if prob is None else prob.astype(np.float64)
    for i in range(n):
        if mask is None or mask[i]:
            labels[i], prob[i], _ = sample_row(z[i], u[i], T, top_k, top_p, min_p)
    return labels, prob
