"""The gated block in f16 where act(G) * U, dG or dU leave f16's range (65,504) and the results do not.

Bounds as in test_gpu_gated.py, with one more: eight neighbouring elements of H, dG or dU (columns 8 i to 8 i + 7 of a row; dU's begin anew) whose largest is m >= 65,520 are held as
multiples of a power of two that brings m to 2^14 or more, so that the smallest spacing there, 2^-24 of f16, is one of at most 2^-38 m: a rounding's absolute part is 2^-39 m.
"""
import ctypes

import numpy as np
import pytest

from oracle import network as N
from test_gpu_gated import ACT_ERROR, D, U, _act, _dev, _empty, _host, _near, _types

pytestmark = pytest.mark.gpu
E, SMALL = U["f16"], D["f16"]
ACTS = ("silu", "gelu", "relu")


def _small(v):
    """The absolute part of the rounding of each element."""
    r, c = v.shape
    wide = np.zeros((r, -(-c // 8), 8))
    wide.reshape(r, -1)[:, :c] = np.abs(v)
    top = np.repeat(wide.max(2), 8, 1)[:, :c]
    return np.where(top >= 65_000, np.maximum(2.0 ** -39 * top, SMALL), SMALL)


def _forward_data(r, p, f, c, seed, extra=0, offset=0, size=300.0):
    """Every fifth row is `size` times as large, and so are G and U of some columns."""
    rng = np.random.default_rng(seed)
    x, gate, up, down = rng.standard_normal((r, p)), rng.standard_normal((p, f)) / p ** 0.5, rng.standard_normal((p, f)) / p ** 0.5, 5e-4 * rng.standard_normal((f, c)) / f ** 0.5
    x[::5] *= size
    cols = rng.choice(f, max(1, f // 40), replace=False)
    gate[:, cols] *= 20.0
    up[:, cols] *= 20.0
    import torch
    return [_dev(a, torch.float16, a.shape[1] + extra, offset) for a in (x, gate, up, down)]


def _check_forward(act, x, gate, up, down, y):
    X, WG, WU, WD = (_host(t) for t in (x, gate, up, down))
    Y, G, UU, H = N.gated_forward(act, X, WG, WU, WD)
    assert np.abs(Y).max() < 65_000
    k1, k2 = X.shape[1] * 2.0 ** -23, H.shape[1] * 2.0 ** -23
    off_g, off_u = k1 * (np.abs(X) @ np.abs(WG)), k1 * (np.abs(X) @ np.abs(WU))
    off_h = np.abs(N.act(act, G)[0]) * off_u + 1.2 * off_g * np.abs(UU) + ACT_ERROR * np.abs(H)
    off = E * np.abs(H) + _small(H) + 2 * off_h
    _near(y, Y, E * np.abs(Y) + SMALL + 2 * (off @ np.abs(WD)) + k2 * (np.abs(H) @ np.abs(WD)), "y")
    return H


def _backward_data(r, p, f, c, seed, extra=0, offset=0):
    """dY, X, Wg, Wu, Wd, G, U: some rows and columns of G and U are large; X and the projections are small, so that the gradients stay in range."""
    import torch
    rng = np.random.default_rng(seed)
    n = rng.standard_normal
    dy, x, gate, up, down, g, u = 1e-4 * n((r, c)), 1e-3 * n((r, p)), 1e-3 * n((p, f)), 1e-3 * n((p, f)), np.clip(2e4 * n((f, c)), -6e4, 6e4), n((r, f)), n((r, f))
    cols = rng.choice(f, max(1, f // 40), replace=False)
    for t in (g, u):
        t[::7] *= 200.0
        t[:, cols] *= 200.0
        np.clip(t, -4e3, 4e3, out=t)
    return [_dev(a, torch.float16, a.shape[1] + extra, offset) for a in (dy, x, gate, up, down, g, u)]


def _check_backward(act, dy, x, gate, up, down, g, u, dx, dgate, dup, ddown):
    DY, X, WG, WU, WD, G, UU = (_host(t) for t in (dy, x, gate, up, down, g, u))
    w = N.gated_backward(act, DY, X, WG, WU, WD, G, UU)
    assert all(np.abs(w[k]).max() < 65_000 for k, t in (("dx", dx), ("dgate", dgate), ("dup", dup), ("ddown", ddown)) if t is not None)
    A = np.abs
    a, da = N.act(act, G)
    off_dh = DY.shape[1] * 2.0 ** -23 * (A(DY) @ A(WD.T))
    off_dg = E * A(w["dg"]) + _small(w["dg"]) + 2 * (A(UU * da) * off_dh + ACT_ERROR * (1 + A(G)) * A(w["dh"] * UU))
    off_du = E * A(w["du"]) + _small(w["du"]) + 2 * (A(a) * off_dh + ACT_ERROR * A(w["du"]))
    off_h = E * A(w["h"]) + _small(w["h"]) + 2 * ACT_ERROR * A(w["h"])
    kf, kr = 2 * WG.shape[1] * 2.0 ** -23, X.shape[0] * 2.0 ** -23
    _near(dx, w["dx"], E * A(w["dx"]) + SMALL + off_dg @ A(WG.T) + off_du @ A(WU.T) + kf * (A(w["dg"]) @ A(WG.T) + A(w["du"]) @ A(WU.T)), "dx")
    _near(dgate, w["dgate"], E * A(w["dgate"]) + SMALL + A(X.T) @ (off_dg + kr * A(w["dg"])), "dgate")
    _near(dup, w["dup"], E * A(w["dup"]) + SMALL + A(X.T) @ (off_du + kr * A(w["du"])), "dup")
    if ddown is not None:
        _near(ddown, w["ddown"], E * A(w["ddown"]) + SMALL + (off_h + kr * A(w["h"])).T @ A(DY), "ddown")
    return w


def _results(r, p, f, c, ld=0):
    import torch
    return [_empty(a, b, torch.float16, b + ld) for a, b in ((r, p), (p, f), (p, f), (f, c))]


SHAPES = [(1, 40, 64, 8), (1, 256, 1000, 130), (3, 64, 70, 65), (16, 64, 1024, 24), (20, 128, 333, 77), (33, 100, 200, 130), (130, 72, 136, 264), (300, 65, 129, 40), (777, 123, 365, 130)]


@pytest.mark.parametrize("r,p,f,c", SHAPES)
@pytest.mark.parametrize("extra,offset", [(0, 0), (3, 1)])
def test_results_are_finite_where_what_lies_between_is_not_in_range(r, p, f, c, extra, offset):
    import torch
    import paper_2312_08728_amd as B
    act = ACTS[(r + p + f) % 3]
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_F16, activation=_act(act)) as block:
        x, gate, up, down = _forward_data(r, p, f, c, r + f, extra, offset)
        y, g, u = (_empty(r, n, torch.float16) for n in (c, f, f))
        for kept in ((g, u), (None, None)):
            block.forward(x, gate, up, down, y, *kept)
            h = _check_forward(act, x, gate, up, down, y)
        assert np.abs(h).max() > 65_520
        data = _backward_data(r, p, f, c, r + f, extra, offset)
        out = _results(r, p, f, c)
        block.backward(*data, *out)
        w = _check_backward(act, *data, *out)
        assert max(np.abs(w[k]).max() for k in ("h", "dg", "du")) > 65_520


@pytest.mark.parametrize("shares", [1, 3])
@pytest.mark.parametrize("tile,rows", [(0, (1, 300, 520)), (1, (5, 130, 257)), (2, (5, 130, 257)), (3, (1, 63, 200)), (4, (1, 17, 32)), (5, (1, 7, 16))])
def test_every_kind_of_tile(tile, rows, shares):
    import torch
    import paper_2312_08728_amd as B
    for i, (r, (p, f, c)) in enumerate(zip(rows, ((200, 264, 136), (512, 320, 700), (333, 517, 65)))):
        act = ACTS[i]
        for extra, offset in ((0, 0), (5, 1)):
            x, gate, up, down = _forward_data(r, p, f, c, 100 + i, extra, offset)
            data = _backward_data(r, p, f, c, 200 + i, extra, offset)
            with B.GatedBlock(p, f, c, r, dtype=B.BMGD_F16, activation=_act(act)) as block:
                assert B.lib.bmgd_internal_gated_tile(ctypes.c_void_p(block.h), tile, shares) == B.BMGD_OK
                y, out = _empty(r, c, torch.float16), _results(r, p, f, c)
                block.forward(x, gate, up, down, y)
                _check_forward(act, x, gate, up, down, y)
                block.backward(*data, *out)
                _check_backward(act, *data, *out)


@pytest.mark.parametrize("r", [5, 200])
def test_a_call_in_range_gives_the_same_bits_before_and_after_one_that_is_not(r):
    """And the rows of a call that are in range the bits that they have beside others that are."""
    import torch
    import paper_2312_08728_amd as B
    p, f, c = 64, 200, 72
    large = _forward_data(r, p, f, c, 1)
    normal = [large[0].clone(), *large[1:]]
    normal[0][::5] /= 300.0
    large[1].mul_(0.3)                                         # (both calls have one set of weights, and ordinary rows are in range)
    back = _backward_data(r, p, f, c, 2)
    tame = [t.clone() for t in back]
    for i in (5, 6):
        tame[i].clamp_(-3.0, 3.0)
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_F16) as block:
        def forward(data):
            y = _empty(r, c, torch.float16)
            block.forward(*data, y)
            return y

        def backward(data):
            out = _results(r, p, f, c)
            block.backward(*data, *out)
            return out

        first, grads = forward(normal), backward(tame)
        again = [forward(large), forward(normal), forward(normal)]
        assert torch.equal(again[1], first) and torch.equal(again[2], first)
        ordinary = torch.arange(r, device="cuda") % 5 != 0
        assert torch.equal(again[0][ordinary], first[ordinary])
        _check_forward("silu", *large, again[0])
        for _ in range(2):
            _check_backward("silu", *back, *backward(back))
            assert all(torch.equal(a, b) for a, b in zip(backward(tame), grads)) and torch.equal(forward(normal), first)
            assert torch.equal(forward(large), again[0])
            dx = _empty(r, p, torch.float16)
            block.backward(*back, dx=dx)
            _check_backward("silu", *back, dx, *backward(back)[1:])                 # (alone its sums may be shared otherwise)
            assert torch.equal(forward(normal), first)
            block.backward(*back)                              # (nothing is wanted: nobody reads what this one leaves)
            assert all(torch.equal(a, b) for a, b in zip(backward(tame), grads)) and torch.equal(forward(normal), first)


def test_a_captured_call_that_is_in_range_at_one_replay_and_not_at_the_next():
    import torch
    import paper_2312_08728_amd as B
    r, p, f, c = 50, 64, 200, 72
    large = _forward_data(r, p, f, c, 1)
    x, weights = large[0].clone(), large[1:]
    y, s = _empty(r, c, torch.float16), torch.cuda.Stream()
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_F16) as block:
        block.forward(x, *weights, y, stream=s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            block.forward(x, *weights, y, stream=s)
        for i in range(8):
            x.copy_(large[0] * (1.0 if i & 1 else 0.003))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            _check_forward("silu", x, *weights, y)
            if i & 2:
                want = _empty(r, c, torch.float16)
                block.forward(x, *weights, want)
                torch.cuda.synchronize()
                assert torch.equal(y, want)


@pytest.mark.parametrize("r", [1, 40, 300])
def test_the_largest_that_f16_gates_can_make(r):
    """act(G) U of 60,000 each, 3.6e9, beside elements of every smaller size, in rows whose weights pick them out one by one: an element is off by no more than 2^-39 of the largest
    of its eight, and those of other eights are as exact as ever."""
    import torch
    import paper_2312_08728_amd as B
    f = 64
    gates = torch.full((f,), 60_000.0)
    gates[8:] = torch.logspace(-2, 4.7, f - 8)
    gate, up = gates.reshape(1, f).half().cuda(), gates.reshape(1, f).half().cuda()
    x = torch.ones(r, 1, dtype=torch.float16, device="cuda")
    down = torch.diag(1.0 / (gates * gates).clamp(min=1.0)).half().cuda()
    down[:8] = 0.0
    down[range(8), range(8)] = 2.0 ** -20
    with B.GatedBlock(1, f, f, r, dtype=B.BMGD_F16, activation=B.BMGD_ACT_RELU) as block:
        y = _empty(r, f, torch.float16)
        block.forward(x, gate, up, down, y)
        h = _check_forward("relu", x, gate, up, down, y)
        assert h.max() > 3e9 and (y[:, 0] > 3_000).all()


@pytest.mark.parametrize("r", [2, 40, 200])
def test_what_is_not_finite_stays_what_it_is_beside_what_is_too_large(r):
    import torch
    import paper_2312_08728_amd as B
    p, f, c = 64, 200, 72
    x, gate, up, down = _forward_data(r, p, f, c, 1, size=30.0)
    for t in (gate, up, down):
        t.abs_()
    x.abs_()
    down[17, 7] = float("inf")                                 # all terms are positive: this column is infinite in every row
    x[1, 3] = float("nan")
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_F16) as block:
        y = _empty(r, c, torch.float16)
        block.forward(x, gate, up, down, y)
        rows, cols = torch.arange(r, device="cuda") != 1, torch.arange(c, device="cuda") != 7
        assert torch.isnan(y[1]).all() and torch.isfinite(y[rows][:, cols]).all() and (y[rows][:, 7] == float("inf")).all()
        y2 = _empty(r, c, torch.float16)
        x[1, 3], down[17, 7] = 0.0, 0.0
        block.forward(x, gate, up, down, y2)
        _check_forward("silu", x, gate, up, down, y2)
        assert torch.equal(y[rows][:, cols], y2[rows][:, cols])


@pytest.mark.parametrize("r,p,f,c", [(20_000, 24, 40, 16), (70, 8, 17_000, 24), (33_000, 16, 24, 8)])
def test_long_sums(r, p, f, c):
    """What is too large lies anywhere along sums of more than 16,384."""
    import torch
    import paper_2312_08728_amd as B
    x, gate, up, down = _forward_data(r, p, f, c, 1)
    data = _backward_data(r, p, f, c, 2)
    less = [0.1 * data[0], *data[1:]]                          # (dWd, of so many rows, in range)
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_F16) as block:
        y, out = _empty(r, c, torch.float16), _results(r, p, f, c)
        block.forward(x, gate, up, down, y)
        _check_forward("silu", x, gate, up, down, y)
        block.backward(*less, *out)
        assert np.abs(_check_backward("silu", *less, *out)["h"]).max() > 65_520
        block.backward(*data, *out[:3])
        w = _check_backward("silu", *data, *out[:3], None)
        assert min(np.abs(w[k]).max() for k in ("dg", "du")) > 65_520


@pytest.mark.parametrize("r", [5, 50])
def test_a_captured_training_step_that_leaves_the_range_at_some_replays(r):
    """Forward and backward in one graph, G and U from the one to the other; other calls on the block in between."""
    import torch
    import paper_2312_08728_amd as B
    p, f, c = 64, 200, 72
    rng = np.random.default_rng(r)
    x, gate, up, down, dy = (_dev(a, torch.float16) for a in (rng.standard_normal((r, p)), rng.standard_normal((p, f)), rng.standard_normal((p, f)), 1e-3 * rng.standard_normal((f, c)),
                                                              1e-3 * rng.standard_normal((r, c))))
    y, g, u = (_empty(r, n, torch.float16) for n in (c, f, f))
    out, s = _results(r, p, f, c), torch.cuda.Stream()
    sizes = [1.0, 100.0, 1.0, 30.0, 100.0, 100.0, 1.0, 1.0]
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_F16) as block:
        def step(stream=None):
            block.forward(x, gate, up, down, y, g, u, stream=stream)
            block.backward(dy, x, gate, up, down, g, u, *out, stream=stream)

        first = x.clone()
        want = []
        for size in sizes:
            x.copy_(first * size)
            step()
            torch.cuda.synchronize()
            want.append([t.clone() for t in (y, g, u, *out)])
            _check_forward("silu", x, gate, up, down, y)
        step(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(s)
        for i, size in enumerate(sizes):
            x.copy_(first * size)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((y, g, u, *out), want[i]))
            if i % 3 == 0:
                step()
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip((y, g, u, *out), want[i]))
