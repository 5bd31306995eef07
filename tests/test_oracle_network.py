"""The plain forms of the gated block and of the AdamW step are pinned before anything is compared with them: gradients by differences, codes by brute
force, the step by a hand-unrolled run."""
import numpy as np
import pytest

from oracle import network as N


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
def test_derivative_of_the_activation_against_differences(name):
    g = np.concatenate([np.linspace(-8, 8, 97) + 0.013, [30.0, -30.0]])
    e = 1e-6
    num = (N.act(name, g + e)[0] - N.act(name, g - e)[0]) / (2 * e)
    assert np.allclose(N.act(name, g)[1], num, atol=1e-8)


def test_activation_values():
    assert N.act("silu", 1.0)[0] == pytest.approx(1 / (1 + np.exp(-1)), rel=1e-15)
    assert N.act("gelu", 1.0)[0] == pytest.approx(0.8413447460685429, rel=1e-14)
    assert N.act("relu", np.array([-2.0, 0.0, 3.0]))[0].tolist() == [0.0, 0.0, 3.0]
    assert N.act("relu", np.array([-2.0, 0.0, 3.0]))[1].tolist() == [0.0, 0.0, 1.0]


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("r,p,f,c", [(1, 1, 1, 1), (3, 5, 4, 2), (6, 2, 7, 3)])
def test_gradients_of_the_block_against_differences(name, r, p, f, c):
    rng = np.random.default_rng(1)
    x, gate, up, down = rng.standard_normal((r, p)), rng.standard_normal((p, f)), rng.standard_normal((p, f)), rng.standard_normal((f, c))
    dy = rng.standard_normal((r, c))
    loss = lambda *a: float(np.sum(dy * N.gated_forward(name, *a)[0]))  # noqa: E731
    _, g, u, _ = N.gated_forward(name, x, gate, up, down)
    got = N.gated_backward(name, dy, x, gate, up, down, g, u)
    for i, k in enumerate(("dx", "dgate", "dup", "ddown")):
        args = [x, gate, up, down]
        num = np.zeros_like(args[i])
        for at in np.ndindex(num.shape):
            both = []
            for e in (1e-6, -1e-6):
                moved = [a.copy() for a in args]
                moved[i][at] += e
                both.append(loss(*moved))
            num[at] = (both[0] - both[1]) / 2e-6
        assert np.allclose(got[k], num, atol=1e-7, rtol=1e-7), k


def test_adamw_first_steps_by_hand():
    th, m, s = N.adamw(np.array([2.0]), np.array([0.5]), np.zeros(1), np.zeros(1), 1, 0.1, 0.9, 0.99, 0.0, 0.5)
    # the first bias-corrected step is the gradient's sign
    assert m == pytest.approx(0.05) and s == pytest.approx(0.0025) and th == pytest.approx(2.0 * 0.95 - 0.1)
    th2, m2, s2 = N.adamw(th, np.array([-1.0]), m, s, 2, 0.1, 0.9, 0.99, 0.0, 0.5)
    mh, sh = (0.9 * 0.05 - 0.1) / (1 - 0.81), (0.99 * 0.0025 + 0.01) / (1 - 0.9801)
    assert th2 == pytest.approx(th * 0.95 - 0.1 * mh / np.sqrt(sh))


def test_codes_are_the_nearest_on_their_scale():
    rng = np.random.default_rng(2)
    m = rng.standard_normal(600) * np.exp(rng.uniform(-12, 0, 600))
    code, top = N.code_m(m)
    roots = np.sqrt(np.abs(m) / np.repeat(top, 256)[:600])
    best = np.argmin(np.abs(roots[:, None] - np.arange(128)[None] / 127.0), axis=1)
    assert np.array_equal(np.abs(code), best) and np.all(np.sign(code) * np.sign(m) >= 0)
    s = m * m
    code, top = N.code_s(s)
    roots = (s / np.repeat(top, 256)[:600]) ** 0.25
    best = np.maximum(1, np.argmin(np.abs(roots[:, None] - np.arange(256)[None] / 255.0), axis=1))
    assert np.array_equal(code, best)
    # a value taken through its code is off by no more than half a step of the root, and a second time stays
    back = N.value_m(*N.code_m(m))
    assert np.max(np.abs(np.sqrt(np.abs(back)) - np.sqrt(np.abs(m))) / np.sqrt(np.repeat(N.code_m(m)[1], 256)[:600])) <= 0.5 / 127 + 1e-12
    assert np.array_equal(N.code_m(back)[0], N.code_m(m)[0])


def test_codes_of_nothing_and_of_the_smallest():
    code, top = N.code_s(np.array([0.0, 1e-30, 1.0]))
    assert code.tolist() == [0, 1, 255] and top.tolist() == [1.0]
    code, top = N.code_m(np.full(5, 1e-39))
    assert code.tolist() == [0] * 5 and top.tolist() == [0.0]
