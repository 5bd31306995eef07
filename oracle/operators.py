"""Plain 64-bit forms of the norm, the 8-bit product and the log probabilities, from their definitions; used by the tests only."""
from __future__ import annotations

import numpy as np

LEAST = 2.0 ** -118


def norm(s, w, eps):
    """(y, 1 / root mean square)."""
    r = 1.0 / np.sqrt((s * s).mean(1) + eps)
    return s * w * r[:, None], r


def codes_of(v):
    """(codes, largest) of the rows of v: v = largest / 127 * code."""
    top = np.abs(v).max(1)
    bad = ~np.isfinite(v).all(1)
    held = ~bad & (top >= LEAST)
    inv = np.where(held, 1.0 / np.where(held, top, 1.0) * 127.0, 0.0)
    codes = np.rint(np.where(bad[:, None], 0.0, v) * inv[:, None]).astype(np.int64)
    return codes, np.where(bad, np.nan, np.where(held, top, 0.0))


def norm_backward(dy, s, w, r, dsum=0.0):
    """(dx, dw)."""
    r = r[:, None]
    along = (w * dy * s).mean(1, keepdims=True)
    return r * (w * dy - s * r * r * along) + dsum, (dy * s * r).sum(0)


def log_probabilities(x):
    """(ln p, entropy) of rows of logits."""
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(1, keepdims=True)
        empty = (m == -np.inf)[:, 0]
        bad = np.isnan(x).any(1) | (m == np.inf)[:, 0]
        e = np.exp(x - np.where(np.isfinite(m), m, 0.0))
        total = e.sum(1, keepdims=True)
        logp = x - m - np.log(total)
        p = e / total
        entropy = -np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0).sum(1)
    logp[empty], entropy[empty] = -np.inf, 0.0
    logp[bad], entropy[bad] = np.nan, np.nan
    return logp, entropy


def best(x, top):
    """Classes in falling order of their logits, the lowest of equal ones first, NaN before all."""
    key = np.where(np.isnan(x), np.inf, x)
    order = np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -key, ~np.isnan(x)), axis=1)
    return order[:, :top]


def logits_gradient(x, labels, dlogprob, dentropy):
    """Gradient of sum dlogprob ln p_label + dentropy H."""
    rows, classes = x.shape
    logp, entropy = log_probabilities(x)
    p = np.exp(logp)
    dl = np.where(labels < 0, 0.0, np.where(labels >= classes, np.nan, dlogprob))
    d = -p * dl[:, None] - dentropy[:, None] * np.where(p > 0, p * (np.where(p > 0, logp, 0.0) + entropy[:, None]), 0.0)
    here = (labels >= 0) & (labels < classes)
    d[np.arange(rows)[here], labels[here]] += dl[here]
    empty = (x == -np.inf).all(1)
    d[empty & (labels < classes)] = 0.0
    d[np.isnan(logp).any(1)] = np.nan
    return d
