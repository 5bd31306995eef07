"""The gated block on up to eight rows, where H, dG and dU keep what their roundings leave: results are off by their own rounding and by what 32 bits add, not by the roundings of
the operands in between.

Bounds: as in test_gpu_gated.py, with u^2 |a_k| + d (two roundings, one behind the other) in the place of u |a_k| + d.
"""
import ctypes

import numpy as np
import pytest

from oracle import network as N
from test_gpu_gated import ACT_ERROR, D, U, _act, _data, _dev, _empty, _host, _near, _types

pytestmark = pytest.mark.gpu


def _check(kind, act, x, gate, up, down, y, dy, g, u, dx, dgate, dup, ddown):
    e, d, A = U[kind], D[kind], np.abs
    X, WG, WU, WD, DY, G, UU = (_host(t) for t in (x, gate, up, down, dy, g, u))
    Y, G0, U0, H = N.gated_forward(act, X, WG, WU, WD)
    k1, kf, kr = X.shape[1] * 2.0 ** -23, H.shape[1] * 2.0 ** -23, 16 * 2.0 ** -23
    off_g, off_u = k1 * (A(X) @ A(WG)), k1 * (A(X) @ A(WU))
    off = e * e * A(H) + d + 2 * (A(N.act(act, G0)[0]) * off_u + 1.2 * off_g * A(U0) + ACT_ERROR * A(H))
    _near(y, Y, e * A(Y) + d + 2 * (off @ A(WD)) + kf * (A(H) @ A(WD)) + 2.0 ** -126, "y")
    w = N.gated_backward(act, DY, X, WG, WU, WD, G, UU)
    a, da = N.act(act, G)
    off_dh = DY.shape[1] * 2.0 ** -23 * (A(DY) @ A(WD.T))
    off_dg = e * e * A(w["dg"]) + d + 2 * (A(UU * da) * off_dh + ACT_ERROR * (1 + A(G)) * A(w["dh"] * UU))
    off_du = e * e * A(w["du"]) + d + 2 * (A(a) * off_dh + ACT_ERROR * A(w["du"]))
    off_h = e * e * A(w["h"]) + d + 2 * ACT_ERROR * A(w["h"])
    _near(dx, w["dx"], e * A(w["dx"]) + d + off_dg @ A(WG.T) + off_du @ A(WU.T) + 2 * kf * (A(w["dg"]) @ A(WG.T) + A(w["du"]) @ A(WU.T)) + 2.0 ** -126, "dx")
    _near(dgate, w["dgate"], e * A(w["dgate"]) + d + A(X.T) @ (off_dg + kr * A(w["dg"])) + 2.0 ** -126, "dgate")
    _near(dup, w["dup"], e * A(w["dup"]) + d + A(X.T) @ (off_du + kr * A(w["du"])) + 2.0 ** -126, "dup")
    _near(ddown, w["ddown"], e * A(w["ddown"]) + d + (off_h + kr * A(w["h"])).T @ A(DY) + 2.0 ** -126, "ddown")


def _run(block, r, p, f, c, kind, act, seed, extra=0, offset=0):
    dtype = _types()[kind][0]
    x, gate, up, down = _data(r, p, f, c, dtype, seed, lds=(p + extra, f + extra, f + extra, c + extra), offset=offset)
    dy = _dev(np.random.default_rng(seed).standard_normal((r, c)), dtype, c + extra, offset)
    y, g, u = (_empty(r, n, dtype, n + extra, offset) for n in (c, f, f))
    out = [_empty(a, b, dtype, b + extra, offset) for a, b in ((r, p), (p, f), (p, f), (f, c))]
    block.forward(x, gate, up, down, y, g, u)
    block.backward(dy, x, gate, up, down, g, u, *out)
    _check(kind, act, x, gate, up, down, y, dy, g, u, *out)
    return y, g, u, *out


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("r,p,f,c", [(1, 1, 1, 1), (1, 8, 8, 8), (1, 37, 19, 5), (1, 512, 2048, 130), (2, 64, 64, 64), (3, 129, 257, 65), (5, 200, 130, 1000), (7, 100, 7, 100),
                                     (8, 1000, 333, 77), (4, 64, 320, 64), (6, 7, 100, 100), (8, 40, 1024, 24), (8, 264, 520, 136)])
@pytest.mark.parametrize("extra,offset", [(0, 0), (3, 1)])
def test_results_are_off_by_their_own_rounding(r, p, f, c, kind, extra, offset):
    import paper_2312_08728_amd as B
    act = ("silu", "gelu", "relu")[(r + p + f) % 3]
    for rows in (r, 100):                                      # a block for so many rows, one for more
        with B.GatedBlock(p, f, c, rows, dtype=_types()[kind][1], activation=_act(act)) as block:
            _run(block, r, p, f, c, kind, act, r + p, extra, offset)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("shares", [1, 3])
@pytest.mark.parametrize("tile", range(6))
def test_every_kind_of_tile(tile, shares, kind):
    """As far as a kind has a form for so few rows."""
    import torch
    import paper_2312_08728_amd as B
    for r, p, f, c in ((1, 200, 264, 136), (6, 512, 320, 700), (8, 333, 517, 65)):
        with B.GatedBlock(p, f, c, 8, dtype=_types()[kind][1]) as block:
            assert B.lib.bmgd_internal_gated_tile(ctypes.c_void_p(block.h), tile, shares) == B.BMGD_OK
            first = _run(block, r, p, f, c, kind, "silu", r)
            again = _run(block, r, p, f, c, kind, "silu", r)
            assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_no_infinity_is_taken_off_an_infinity(kind):
    """Where H is infinite nothing is left beside it: Y is infinite, and the rows around it are what they are."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    for r in (1, 4, 8):
        x = torch.ones(r, 1, dtype=dtype, device="cuda")
        x[r // 2] = float("inf")
        one = torch.full((1, 64), 0.5, dtype=dtype, device="cuda")
        down = torch.full((64, 8), 0.25, dtype=dtype, device="cuda")
        with B.GatedBlock(1, 64, 8, r, dtype=code, activation=B.BMGD_ACT_RELU) as block:
            y, g, u = (_empty(r, n, dtype) for n in (8, 64, 64))
            block.forward(x, one, one, down, y, g, u)
            inf = torch.arange(r, device="cuda") == r // 2
            assert (y[inf] == float("inf")).all() and (y[~inf] == 4.0).all()
            dy = torch.ones(r, 8, dtype=dtype, device="cuda")
            dx, ddown = _empty(r, 1, dtype), _empty(64, 8, dtype)
            block.backward(dy, x, one, one, down, g, u, dx=dx, ddown=ddown)
            assert (dx[inf] == float("inf")).all() and torch.isfinite(dx[~inf]).all() and (ddown == float("inf")).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("r", [1, 3, 8])
def test_infinite_weights_and_gradients_meet_no_rests(r, kind):
    """All terms positive: what has an infinite weight, or an infinite dY, among its terms is infinite, everything else has the bits that it has without."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    p, f, c = 40, 72, 24
    rng = np.random.default_rng(r)
    x, gate, up, down, dy = (_dev(0.1 + rng.random(s), dtype) for s in ((r, p), (p, f), (p, f), (f, c), (r, c)))
    row = r // 2
    with B.GatedBlock(p, f, c, r, dtype=code, activation=B.BMGD_ACT_RELU) as block:
        def run():
            y, g, u = (_empty(r, n, dtype) for n in (c, f, f))
            out = [_empty(a, b, dtype) for a, b in ((r, p), (p, f), (p, f), (f, c))]
            block.forward(x, gate, up, down, y, g, u)
            block.backward(dy, x, gate, up, down, g0, u0, *out)
            return y, *out

        g0, u0 = (_dev(0.1 + rng.random((r, f)), dtype) for _ in range(2))
        plain = run()
        inf = lambda t: t == float("inf")  # noqa: E731
        at = lambda n, i: torch.arange(n, device="cuda") == i  # noqa: E731
        keep = down[17, 7].clone()
        down[17, 7] = float("inf")                             # Y's column, and dH's: all of dX, columns of dWg and dWu
        y, dx, dgate, dup, ddown = run()
        assert inf(y[:, 7]).all() and torch.equal(y[:, ~at(c, 7)], plain[0][:, ~at(c, 7)])
        assert inf(dx).all() and inf(dgate[:, 17]).all() and inf(dup[:, 17]).all() and torch.equal(dgate[:, ~at(f, 17)], plain[2][:, ~at(f, 17)])
        assert torch.equal(ddown, plain[4])
        down[17, 7] = keep
        dy[row, 5] = float("inf")
        y, dx, dgate, dup, ddown = run()
        assert inf(dx[row]).all() and torch.equal(dx[~at(r, row)], plain[1][~at(r, row)]) and inf(dgate).all() and inf(dup).all()
        assert inf(ddown[:, 5]).all() and torch.equal(ddown[:, ~at(c, 5)], plain[4][:, ~at(c, 5)]) and torch.equal(y, plain[0])
        x[row, 3] = float("inf")
        dy[row, 5] = 1.0
        y, dx, dgate, dup, ddown = run()
        assert inf(y[row]).all() and torch.equal(y[~at(r, row)], plain[0][~at(r, row)]) and inf(dgate[3]).all() and inf(dup[3]).all()
        assert torch.isfinite(dgate[~at(p, 3)]).all() and torch.isfinite(ddown).all() and torch.isfinite(dx).all()
