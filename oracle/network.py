"""Plain 64-bit forms of the gated block and of the AdamW step, from their definitions; used by the tests only."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 256


def _erf(x):
    return np.vectorize(math.erf, otypes=[np.float64])(x)


def act(name, g):
    """act(g) and act'(g)."""
    g = np.asarray(g, dtype=np.float64)
    if name == "relu":
        return np.where(g > 0, g, 0.0), np.where(g > 0, 1.0, 0.0)
    if name == "silu":
        s = np.where(g >= 0, 1.0 / (1.0 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1.0 + np.exp(-np.abs(g))))
        return g * s, s + g * s * (1.0 - s)
    cdf, pdf = 0.5 * (1.0 + _erf(g / math.sqrt(2.0))), np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    return g * cdf, cdf + g * pdf


def gated_forward(name, x, gate, up, down):
    """(Y, G, U, H)."""
    g, u = x @ gate, x @ up
    h = act(name, g)[0] * u
    return h @ down, g, u, h


def gated_backward(name, dy, x, gate, up, down, g, u):
    """dict of dx, dgate, dup, ddown and what lies between (h, dh, dg, du)."""
    a, da = act(name, g)
    dh = dy @ down.T
    dg, du, h = dh * u * da, dh * a, a * u
    return {"dx": dg @ gate.T + du @ up.T, "dgate": x.T @ dg, "dup": x.T @ du, "ddown": h.T @ dy, "h": h, "dh": dh, "dg": dg, "du": du}


def adamw(theta, g, m, s, k, lr, beta1, beta2, eps, decay, grad_scale=1.0):
    """theta, m, s after the k-th update."""
    g = grad_scale * g
    m = beta1 * m + (1.0 - beta1) * g
    s = beta2 * s + (1.0 - beta2) * g * g
    step = (m / (1.0 - beta1 ** k)) / (np.sqrt(s / (1.0 - beta2 ** k)) + eps)
    return theta * (1.0 - lr * decay) - lr * step, m, s


def _blocks(v):
    pad = -len(v) % BLOCK
    return np.concatenate([v, np.zeros(pad)]).reshape(-1, BLOCK)


def value_m(code, scale):
    c = _blocks(np.asarray(code, dtype=np.float64)) / 127.0
    return (scale[:, None] * c * np.abs(c)).ravel()[: len(code)]


def value_s(code, scale):
    c = _blocks(np.asarray(code, dtype=np.float64)) / 255.0
    return (scale[:, None] * c ** 4).ravel()[: len(code)]


def code_m(m):
    """(codes, scales) of finite first moments."""
    v = _blocks(np.asarray(m, dtype=np.float64))
    top = np.abs(v).max(1)
    top = np.where(top >= 2.0 ** -126, top, 0.0)
    share = np.abs(v) / np.where(top > 0, top, 1.0)[:, None] * (top > 0)[:, None]
    return (np.rint(127.0 * np.sqrt(share)) * np.sign(v)).ravel()[: len(m)].astype(np.int64), top


def code_s(s):
    v = _blocks(np.asarray(s, dtype=np.float64))
    top = v.max(1)
    top = np.where(top >= 2.0 ** -126, top, 0.0)
    share = v / np.where(top > 0, top, 1.0)[:, None] * (top > 0)[:, None]
    code = np.maximum(np.rint(255.0 * share ** 0.25), (share > 0) * 1.0)
    return code.ravel()[: len(s)].astype(np.int64), top
