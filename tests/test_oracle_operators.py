"""The 64-bit forms of norm, product codes and log probabilities: closed forms and differences."""
import numpy as np
import pytest

from oracle import operators as O


def _difference(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_norm_and_its_gradient():
    rng = np.random.default_rng(0)
    s, w, dy, ds = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    y, r = O.norm(s, np.ones(7), 0.0)
    assert np.allclose((y * y).mean(1), 1.0) and np.allclose(y, s * r[:, None])
    r = O.norm(s, w, 1e-3)[1]
    dx, dw = O.norm_backward(dy, s, w, r, ds)
    assert np.allclose(dx, _difference(lambda a: (O.norm(a, w, 1e-3)[0] * dy).sum() + (a * ds).sum(), s), atol=1e-8)
    assert np.allclose(dw, _difference(lambda a: (O.norm(s, a, 1e-3)[0] * dy).sum(), w), atol=1e-8)


def test_codes():
    v = np.array([[127.0, 2.5, 3.5, -0.5, 1.5], [0.0, 0.0, 0.0, 0.0, 0.0], [2.0 ** -119, 0, 0, 0, 0], [np.inf, 1, 2, 3, 4], [np.nan, 1, 2, 3, 4]])
    codes, top = O.codes_of(v)
    assert codes[0].tolist() == [127, 2, 4, 0, 2] and not codes[1:].any()           # half to even
    assert top[:3].tolist() == [127.0, 0.0, 0.0] and np.isnan(top[3:]).all()


@pytest.mark.parametrize("dl,dh", [(1.0, 0.0), (0.0, 1.0), (-0.7, 0.3)])
def test_log_probabilities_and_their_gradient(dl, dh):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(3, 6)) * 2
    x[1, 4:] = -np.inf
    labels = np.array([2, 1, -1])
    logp, entropy = O.log_probabilities(x)
    p = np.exp(logp)
    assert np.allclose(p.sum(1), 1) and np.allclose(O.log_probabilities(np.zeros((1, 8)))[1], np.log(8))

    def value(a):
        lp, h = O.log_probabilities(a)
        return sum(dl * lp[i, c] for i, c in enumerate(labels) if c >= 0) + dh * h.sum()
    d = O.logits_gradient(x, labels, np.full(3, dl), np.full(3, dh))
    finite = np.isfinite(x)
    flat = x[finite]

    def of_flat(f):
        a = x.copy()
        a[finite] = f
        return value(a)
    assert np.allclose(d[finite], _difference(of_flat, flat), atol=1e-8) and not d[~finite].any()


def test_rows_without_a_distribution():
    x = np.array([[-np.inf] * 3, [np.nan, 1, 2], [np.inf, 0, 0]])
    logp, entropy = O.log_probabilities(x)
    assert (logp[0] == -np.inf).all() and entropy[0] == 0 and np.isnan(logp[1:]).all() and np.isnan(entropy[1:]).all()
    d = O.logits_gradient(x, np.array([1, 1, 1]), np.ones(3), np.ones(3))
    assert not d[0].any() and np.isnan(d[1:]).all()
    d = O.logits_gradient(np.zeros((1, 3)), np.array([3]), np.ones(1), np.zeros(1))
    assert np.isnan(d).all()


def test_order_of_equal_logits():
    x = np.array([[1.0, 3.0, 3.0, -0.0, 0.0], [np.nan, 2.0, np.inf, np.nan, 2.0]])
    assert O.best(x, 5).tolist() == [[1, 2, 0, 3, 4], [0, 3, 2, 1, 4]]
