"""The gated block's kernels against the plain form in 64 bits, element by element.

Bounds.  u is the largest relative error of a rounding to the type (2^-8 for bf16, 2^-11 for f16), d the largest absolute one below its normal range
(2^-134, 2^-25).  A result r = sum of a_k b_k whose operands a_k were rounded from fp32 is off by at most
    u |r| + d                       its own rounding
  + sum (u |a_k| + d) |b_k|         those of the operands
  + (K 2^-23) sum |a_k b_k|         K additions in fp32
and by what the operands inherit: the activation is good to 2^-19 of its value (hardware exponential and reciprocal, erf), and dH's own sum comes first.
The sum of all these is what is allowed, times 1.01.
"""
import numpy as np
import pytest

from oracle import network as N

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
D = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}
ACT_ERROR = 2.0 ** -19


def _types():
    import torch
    import paper_2312_08728_amd as B
    return {"bf16": (torch.bfloat16, B.BMGD_BF16), "f16": (torch.float16, B.BMGD_F16)}


def _act(name):
    import paper_2312_08728_amd as B
    return {"silu": B.BMGD_ACT_SILU, "gelu": B.BMGD_ACT_GELU, "relu": B.BMGD_ACT_RELU}[name]


def _dev(a, dtype, ld=None, offset=0):
    """a on the device, rows `ld` elements apart, the first one `offset` elements into its allocation; the rest of it is NaN."""
    import torch
    r, c = a.shape
    ld = c if ld is None else ld
    flat = torch.full((offset + max(0, r - 1) * ld + c if r else offset + 1,), float("nan"), dtype=dtype, device="cuda")
    t = flat[offset:].as_strided((r, c), (ld, 1)) if r else flat[:0].reshape(0, c)
    if r:
        t.copy_(torch.from_numpy(a))
    return t


def _host(t):
    return t.double().cpu().numpy()


def _data(r, p, f, c, dtype, seed, lds=(None,) * 4, offset=0):
    rng = np.random.default_rng(seed)
    x, gate, up, down = rng.standard_normal((r, p)), rng.standard_normal((p, f)) / p ** 0.5, rng.standard_normal((p, f)) / p ** 0.5, rng.standard_normal((f, c)) / f ** 0.5
    return [_dev(a, dtype, ld, offset) for a, ld in zip((x, gate, up, down), lds)]


def _near(got, want, allowed, what):
    got = _host(got)
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= 1.01 * allowed)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / allowed):.2f} of what is allowed at {np.argwhere(bad)[0]}"


def _check_forward(kind, act, x, gate, up, down, y, g=None, u=None):
    e, d = U[kind], D[kind]
    X, WG, WU, WD = (_host(t) for t in (x, gate, up, down))
    Y, G, UU, H = N.gated_forward(act, X, WG, WU, WD)
    k1, k2 = X.shape[1] * 2.0 ** -23, H.shape[1] * 2.0 ** -23
    off_g, off_u = k1 * (np.abs(X) @ np.abs(WG)), k1 * (np.abs(X) @ np.abs(WU))
    if g is not None:
        _near(g, G, e * np.abs(G) + d + 2 * off_g, "g")
        _near(u, UU, e * np.abs(UU) + d + 2 * off_u, "u")
    a, da = N.act(act, G)
    off_h = np.abs(a) * off_u + 1.2 * off_g * np.abs(UU) + ACT_ERROR * np.abs(H)       # (|act'| is at most 1.13)
    off = e * np.abs(H) + d + 2 * off_h
    _near(y, Y, e * np.abs(Y) + d + 2 * (off @ np.abs(WD)) + k2 * (np.abs(H) @ np.abs(WD)) + 2.0 ** -126, "y")


def _check_backward(kind, act, dy, x, gate, up, down, g, u, dx, dgate, dup, ddown):
    e, d = U[kind], D[kind]
    DY, X, WG, WU, WD, G, UU = (_host(t) for t in (dy, x, gate, up, down, g, u))
    w = N.gated_backward(act, DY, X, WG, WU, WD, G, UU)
    a, da = N.act(act, G)
    off_dh = DY.shape[1] * 2.0 ** -23 * (np.abs(DY) @ np.abs(WD.T))
    # the derivative is a sum of terms of up to 1 + |g|, so its error is one of those
    off_dg = e * np.abs(w["dg"]) + d + 2 * (np.abs(UU * da) * off_dh + ACT_ERROR * (1 + np.abs(G)) * np.abs(w["dh"] * UU))
    off_du = e * np.abs(w["du"]) + d + 2 * (np.abs(a) * off_dh + ACT_ERROR * np.abs(w["du"]))
    off_h = e * np.abs(w["h"]) + d + 2 * ACT_ERROR * np.abs(w["h"])
    kf, kr = 2 * WG.shape[1] * 2.0 ** -23, X.shape[0] * 2.0 ** -23
    A = np.abs
    if dx is not None:
        _near(dx, w["dx"], e * A(w["dx"]) + d + off_dg @ A(WG.T) + off_du @ A(WU.T) + kf * (A(w["dg"]) @ A(WG.T) + A(w["du"]) @ A(WU.T)) + 2.0 ** -126, "dx")
    if dgate is not None:
        _near(dgate, w["dgate"], e * A(w["dgate"]) + d + A(X.T) @ (off_dg + kr * A(w["dg"])) + 2.0 ** -126, "dgate")
        _near(dup, w["dup"], e * A(w["dup"]) + d + A(X.T) @ (off_du + kr * A(w["du"])) + 2.0 ** -126, "dup")
    if ddown is not None:
        _near(ddown, w["ddown"], e * A(w["ddown"]) + d + (off_h + kr * A(w["h"])).T @ A(DY) + 2.0 ** -126, "ddown")


def _empty(rows, cols, dtype, ld=None, offset=0):
    import torch
    ld = cols if ld is None else ld
    return torch.full((offset + rows * ld + 8,), 7.0, dtype=dtype, device="cuda")[offset:].as_strided((rows, cols), (ld, 1))


SHAPES = [
    (1, 1, 1, 1), (1, 8, 8, 8), (1, 37, 19, 5), (2, 64, 64, 64), (1, 512, 1000, 130), (3, 129, 257, 65), (5, 200, 130, 1000), (8, 1000, 333, 77),
    (9, 64, 320, 64), (16, 40, 1024, 24), (17, 1024, 72, 200), (33, 100, 200, 130), (64, 64, 64, 64), (65, 72, 136, 264), (100, 200, 600, 130),
    (127, 123, 131, 130), (256, 256, 128, 256), (257, 136, 264, 520), (300, 65, 63, 1), (777, 123, 365, 130), (1000, 8, 16, 8),
]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("r,p,f,c", SHAPES)
def test_forward_and_backward_at_many_sizes(r, p, f, c, kind):
    import paper_2312_08728_amd as B
    act = ("silu", "gelu", "relu")[(r + p + f) % 3]
    dtype, code = _types()[kind]
    x, gate, up, down = _data(r, p, f, c, dtype, seed=r + p)
    with B.GatedBlock(p, f, c, r, dtype=code, activation=_act(act)) as block:
        y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
        block.forward(x, gate, up, down, y, g, u)
        _check_forward(kind, act, x, gate, up, down, y, g, u)
        only = _empty(r, c, dtype)
        block.forward(x, gate, up, down, only)
        assert (only == y).all()
        dy = _dev(np.random.default_rng(r).standard_normal((r, c)), dtype)
        out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
        block.backward(dy, x, gate, up, down, g, u, *out)
        _check_backward(kind, act, dy, x, gate, up, down, g, u, *out)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("r,p,f,c,extra,offset", [(70, 64, 128, 64, 8, 8), (70, 64, 128, 64, 3, 1), (1, 64, 128, 72, 5, 3), (130, 61, 99, 30, 7, 0), (40, 128, 64, 8, 64, 2)])
def test_rows_apart_and_at_odd_addresses(r, p, f, c, extra, offset, kind):
    """Strided views whose gaps hold NaN: nothing of them may reach a result, and nothing may be written to them."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    x, gate, up, down = _data(r, p, f, c, dtype, 5, lds=(p + extra, f + extra, f + 2 * extra, c + extra), offset=offset)
    with B.GatedBlock(p, f, c, r + 3, dtype=code) as block:
        y, g, u = (_empty(r, n, dtype, n + extra, offset) for n in (c, f, f))
        block.forward(x, gate, up, down, y, g, u)
        _check_forward(kind, "silu", x, gate, up, down, y, g, u)
        dy = _dev(np.random.default_rng(3).standard_normal((r, c)), dtype, c + extra, offset)
        out = [_empty(a, b, dtype, b + extra, offset) for a, b in ((r, p), (p, f), (p, f), (f, c))]
        block.backward(dy, x, gate, up, down, g, u, *out)
        _check_backward(kind, "silu", dy, x, gate, up, down, g, u, *out)
        for t in (y, g, u, *out):
            rows, cols = t.shape
            gaps = t.as_strided((rows, extra), (cols + extra, 1), t.storage_offset() + cols)[: rows - 1]
            assert (gaps == 7.0).all()
    torch.cuda.synchronize()


def test_fewer_rows_than_the_block_was_made_for_and_gradients_left_out():
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    p, f, c = 96, 200, 40
    with B.GatedBlock(p, f, c, 500, dtype=code) as block:
        for r in (500, 3, 1, 77):
            x, gate, up, down = _data(r, p, f, c, dtype, r)
            y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
            block.forward(x, gate, up, down, y, g, u)
            _check_forward("bf16", "silu", x, gate, up, down, y, g, u)
            dy = _dev(np.random.default_rng(r).standard_normal((r, c)), dtype)
            dx, dgate, dup, ddown = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
            block.backward(dy, x, gate, up, down, g, u, dx=dx)
            block.backward(dy, x, gate, up, down, g, u, dgate=dgate, dup=dup)
            block.backward(dy, x, gate, up, down, g, u, ddown=ddown)
            _check_backward("bf16", "silu", dy, x, gate, up, down, g, u, dx, dgate, dup, ddown)


def test_no_rows():
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    p, f, c = 33, 70, 9
    x, gate, up, down = _data(0, p, f, c, dtype, 1)
    with B.GatedBlock(p, f, c, 4, dtype=code) as block:
        y, g = _empty(0, c, dtype), _empty(0, f, dtype)
        block.forward(x, gate, up, down, y, g, g)
        out = [_empty(0, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)]
        block.backward(y, x, gate, up, down, g, g, *out)
        assert all((t == 0).all() for t in out[1:])


@pytest.mark.parametrize("r", [1, 5, 40, 200])
def test_what_is_not_finite_stays_in_its_row_and_column(r):
    """A row of X with NaN or infinity spoils its own results and the weights' gradients only; a weight its own columns."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    p, f, c = 72, 100, 60
    x, gate, up, down = _data(r, p, f, c, dtype, 8)
    x[r // 2, 3] = float("nan")
    down[:, 7] = float("inf")
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
        block.forward(x, gate, up, down, y, g, u)
        keep = torch.ones(r, dtype=torch.bool, device="cuda")
        keep[r // 2] = False
        cols = torch.ones(c, dtype=torch.bool, device="cuda")
        cols[7] = False
        assert torch.isnan(y[r // 2]).all() and torch.isnan(g[r // 2]).all()
        assert torch.isfinite(y[keep][:, cols]).all() and torch.isfinite(g[keep]).all()
        assert not torch.isfinite(y[:, 7]).any()


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_activation_far_out(act):
    """Gates from -1e4 to 1e4 and zero: no overflow on the way."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    gates = torch.tensor([0.0, -0.0, 1e-3, -1e-3, 1, -1, 5, -5, 20, -20, 88, -88, 100, -100, 1e4, -1e4], dtype=dtype, device="cuda")
    f = len(gates)
    gate, up = gates.reshape(1, f).clone(), torch.full((1, f), 2.0, dtype=dtype, device="cuda")
    down = torch.eye(f, dtype=dtype, device="cuda")
    x = torch.ones(1, 1, dtype=dtype, device="cuda")
    with B.GatedBlock(1, f, f, 1, dtype=code, activation=_act(act)) as block:
        y, g, u = _empty(1, f, dtype), _empty(1, f, dtype), _empty(1, f, dtype)
        block.forward(x, gate, up, down, y, g, u)
        _check_forward("bf16", act, x, gate, up, down, y, g, u)
        dy = torch.ones(1, f, dtype=dtype, device="cuda")
        out = _empty(1, 1, dtype), _empty(1, f, dtype), _empty(1, f, dtype), _empty(f, f, dtype)
        block.backward(dy, x, gate, up, down, g, u, *out)
        _check_backward("bf16", act, dy, x, gate, up, down, g, u, *out)


def test_gradients_against_differences():
    """The loss sum(dY * Y), in 64 bits, along random directions against the kernels' gradients: differences of size 1e-4 are off by 1e-7 of
    the loss's third derivative, the gradients by their rounding, at most 3 u of the norm of what they are multiplied with."""
    import paper_2312_08728_amd as B
    dtype, code = _types()["f16"]
    r, p, f, c = 40, 24, 48, 16
    x, gate, up, down = _data(r, p, f, c, dtype, 21)
    dy = _dev(np.random.default_rng(22).standard_normal((r, c)), dtype)
    with B.GatedBlock(p, f, c, r, dtype=code, activation=_act("gelu")) as block:
        y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
        block.forward(x, gate, up, down, y, g, u)
        out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
        block.backward(dy, x, gate, up, down, g, u, *out)
    args, DY = [_host(t) for t in (x, gate, up, down)], _host(dy)
    rng = np.random.default_rng(23)
    for i, grad in enumerate(out):
        for _ in range(4):
            way = rng.standard_normal(args[i].shape)
            side = []
            for e in (1e-4, -1e-4):
                moved = list(args)
                moved[i] = args[i] + e * way
                side.append(np.sum(DY * N.gated_forward("gelu", *moved)[0]))
            num = (side[0] - side[1]) / 2e-4
            have = float(np.sum(_host(grad) * way))
            assert abs(num - have) <= 3 * U["f16"] * np.linalg.norm(_host(grad)) * np.linalg.norm(way) + 1e-5


def test_the_same_call_gives_the_same_bits_also_where_workgroups_share_tiles():
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    for r, p, f, c in ((12, 2048, 96, 128), (4000, 40, 72, 24), (200, 1500, 64, 100), (1, 4000, 100, 64)):
        x, gate, up, down = _data(r, p, f, c, dtype, 31)
        dy = _dev(np.random.default_rng(1).standard_normal((r, c)), dtype)
        with B.GatedBlock(p, f, c, r, dtype=code) as block:
            first = None
            for _ in range(6):
                y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
                out = [_empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)]
                block.forward(x, gate, up, down, y, g, u)
                block.backward(dy, x, gate, up, down, g, u, *out)
                now = [y, g, u, *out]
                assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
                first = now
            _check_forward("bf16", "silu", x, gate, up, down, *first[:3])
            _check_backward("bf16", "silu", dy, x, gate, up, down, *first[1:])


def test_calls_on_several_streams_follow_one_another():
    """Both calls use one workspace: the second, on another stream, waits for the first, which stands behind a busy stream."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, p, f, c = 300, 256, 512, 64
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        sets = [_data(r, p, f, c, dtype, seed) for seed in (1, 2)]
        ys = [_empty(r, c, dtype) for _ in sets]
        torch.cuda.synchronize()
        with torch.cuda.stream(s1):
            for _ in range(20):
                busy = busy @ busy * 1e-3
        block.forward(*sets[0], ys[0], stream=s1)
        block.forward(*sets[1], ys[1], stream=s2)
        block.forward(*sets[0], ys[0], stream=s1)
        torch.cuda.synchronize()
        for data, y in zip(sets, ys):
            _check_forward("bf16", "silu", *data, y)


def test_captured_into_a_graph():
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, p, f, c = 50, 300, 96, 80
    x, gate, up, down = _data(r, p, f, c, dtype, 1)
    y, want = _empty(r, c, dtype), _empty(r, c, dtype)
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        s = torch.cuda.Stream()
        block.forward(x, gate, up, down, y, stream=s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            block.forward(x, gate, up, down, y, stream=s)
        for i in range(4):
            x.copy_(torch.randn(r, p, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            block.forward(x, gate, up, down, want)
            torch.cuda.synchronize()
            assert torch.equal(y, want)
            _check_forward("bf16", "silu", x, gate, up, down, y)


def test_workspace_of_the_caller():
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["f16"]
    cfg = B.bmgd_gated_config(50, 70, 30, 20, code, 0, None, 0)
    need = B.bmgd_gated_workspace_bytes(cfg)
    area = torch.full((need + 512,), 85, dtype=torch.uint8, device="cuda")
    at = -area.data_ptr() % 256
    x, gate, up, down = _data(20, 50, 70, 30, dtype, 4)
    with B.GatedBlock(50, 70, 30, 20, dtype=code, workspace=area[at:at + need]) as block:
        y = _empty(20, 30, dtype)
        block.forward(x, gate, up, down, y)
        _check_forward("f16", "silu", x, gate, up, down, y)
    assert (area[:at] == 85).all() and (area[at + need:] == 85).all()
    with pytest.raises(B.BmgdError):
        B.GatedBlock(50, 70, 30, 20, dtype=code, workspace=area[at:at + need - 256])


def test_refusals():
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    x, gate, up, down = _data(4, 16, 24, 8, dtype, 4)
    y, g = _empty(4, 8, dtype), _empty(4, 24, dtype)
    with B.GatedBlock(16, 24, 8, 4, dtype=code) as block:
        for bad in ((x.float(), gate, up, down, y), (x.cpu(), gate, up, down, y), (x[:, :8], gate, up, down, y), (x, gate[:8], up, down, y),
                    (x, gate, up.t(), down, y), (x, gate, up, down, y[:2]), (x.t().contiguous().t(), gate, up, down, y)):
            with pytest.raises(ValueError):
                block.forward(*bad)
        with pytest.raises(B.BmgdError) as e:
            block.forward(x, gate, up, down, y, g)
        assert e.value.code == B.BMGD_EINVAL and "together" in str(e.value)
        five = _empty(5, 16, dtype)
        with pytest.raises(B.BmgdError) as e:
            block.forward(five, gate, up, down, _empty(5, 8, dtype))
        assert "max_rows" in str(e.value)
        with pytest.raises(B.BmgdError):
            block.backward(y, x, gate, up, down, g, g, dgate=_empty(16, 24, dtype))
        with pytest.raises(B.BmgdError):                       # rows on top of one another
            block.forward(x[:1].expand(4, 16), gate, up, down, y)
        t = B.bmgd_gated_tensors()
        assert B.bmgd_gated_forward(block.h, 4, t) == B.BMGD_EINVAL and "x must not be NULL" in B.bmgd_gated_last_error(block.h)
        assert B.bmgd_gated_forward(block.h, -1, t) == B.BMGD_EINVAL
        assert B.bmgd_gated_forward(block.h, 4, None) == B.BMGD_EINVAL
        block.forward(x, gate, up, down, y)
        _check_forward("bf16", "silu", x, gate, up, down, y)
    torch.cuda.synchronize()


@pytest.mark.parametrize("shares", [1, 3])
@pytest.mark.parametrize("tile,rows", [(0, (1, 300, 520)), (1, (5, 130, 257)), (2, (5, 130, 257)), (3, (1, 63, 200)), (4, (1, 17, 32)), (5, (1, 7, 16))])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_every_kind_of_tile_with_and_without_shared_sums(kind, tile, rows, shares):
    """Sizes that end inside a tile, inside a step of 64 and at their edges, for each tile whatever the block's own choice would be."""
    import ctypes
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    for i, (r, (p, f, c)) in enumerate(zip(rows, ((200, 264, 136), (512, 320, 700), (333, 517, 65)))):
        act = ("silu", "gelu", "relu")[i]
        x, gate, up, down = _data(r, p, f, c, dtype, 100 + i)
        dy = _dev(np.random.default_rng(i).standard_normal((r, c)), dtype)
        with B.GatedBlock(p, f, c, r, dtype=code, activation=_act(act)) as block:
            assert B.lib.bmgd_internal_gated_tile(ctypes.c_void_p(block.h), tile, shares) == B.BMGD_OK
            for _ in range(2):                                 # (counters are zero again after a launch)
                y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
                block.forward(x, gate, up, down, y, g, u)
                _check_forward(kind, act, x, gate, up, down, y, g, u)
                out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
                block.backward(dy, x, gate, up, down, g, u, *out)
                _check_backward(kind, act, dy, x, gate, up, down, g, u, *out)


def test_many_rows_at_the_block_s_own_choice():
    """Enough tiles for the large kind in every product; columns and sums that end inside a tile and a step."""
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, p, f, c = 2_900, 712, 2_056, 1_416
    x, gate, up, down = _data(r, p, f, c, dtype, 3)
    dy = _dev(np.random.default_rng(4).standard_normal((r, c)), dtype)
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
        block.forward(x, gate, up, down, y, g, u)
        _check_forward("bf16", "silu", x, gate, up, down, y, g, u)
        out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
        block.backward(dy, x, gate, up, down, g, u, *out)
        _check_backward("bf16", "silu", dy, x, gate, up, down, g, u, *out)


@pytest.mark.parametrize("stride", [1 << 26, (1 << 26) + 3])
def test_rows_so_far_apart_that_offsets_pass_32_bits(stride):
    """40 rows of 5.4 GB: element offsets beyond 2^31, in place and through the copy."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, p, f, c = 40, 64, 72, 24
    x, gate, up, down = _data(r, p, f, c, dtype, 3)
    far = torch.empty(39 * stride + p, dtype=dtype, device="cuda").as_strided((r, p), (stride, 1))
    far.copy_(x)
    out_far = torch.empty(39 * stride + c, dtype=dtype, device="cuda").as_strided((r, c), (stride, 1))
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        block.forward(far, gate, up, down, out_far)
        _check_forward("bf16", "silu", x, gate, up, down, out_far)
    del far, out_far
    torch.cuda.empty_cache()


def test_unequal_strides_of_the_two_projections():
    import paper_2312_08728_amd as B
    dtype, code = _types()["f16"]
    r, p, f, c = 30, 64, 128, 64
    x, gate, up, down = _data(r, p, f, c, dtype, 5, lds=(None, f + 8, f + 64, None))
    dy = _dev(np.random.default_rng(3).standard_normal((r, c)), dtype)
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
        block.forward(x, gate, up, down, y, g, u)
        _check_forward("f16", "silu", x, gate, up, down, y, g, u)
        dx = _empty(r, p, dtype)
        block.backward(dy, x, gate, up, down, g, u, dx=dx)
        _check_backward("f16", "silu", dy, x, gate, up, down, g, u, dx, None, None, None)


def test_small_half_precision_numbers_are_not_taken_for_zero():
    """Rows far below f16's normal range (6.1e-5), in both directions."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["f16"]
    for r in (1, 40, 300):
        p, f, c = 64, 128, 72
        x, gate, up, down = _data(r, p, f, c, dtype, 6)
        x *= 1e-6
        up *= 1e3
        with B.GatedBlock(p, f, c, r, dtype=code) as block:
            y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
            block.forward(x, gate, up, down, y, g, u)
            _check_forward("f16", "silu", x, gate, up, down, y, g, u)
            assert (g != 0).float().mean() > 0.9 and float(g.abs().max()) < 2e-5
            x *= 1e6
            block.forward(x, gate, up, down, y, g, u)
            dy = _dev(1e-6 * np.random.default_rng(r).standard_normal((r, c)), dtype)
            out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
            block.backward(dy, x, gate, up, down, g, u, *out)
            _check_backward("f16", "silu", dy, x, gate, up, down, g, u, *out)
            assert (out[3] != 0).any()
    torch.cuda.synchronize()


@pytest.mark.parametrize("f", [1, 3, 7, 8, 9, 63, 70, 129])
@pytest.mark.parametrize("r", [3, 200])
def test_an_infinite_gradient_meets_no_zeros_of_columns_that_are_not_there(r, f):
    """All terms positive, one element of dY infinite: the formula has no difference and no product with zero, so its row of dX, all of dWg and dWu and its column of dWd are infinite."""
    import torch
    import paper_2312_08728_amd as B
    p, c = 24, 11
    rng = np.random.default_rng(f)
    x, gate, up, down = (_dev(0.5 + rng.random(s), torch.bfloat16) for s in ((r, p), (p, f), (p, f), (f, c)))
    g, u = (_dev(0.5 + rng.random((r, f)), torch.bfloat16, ld=f + 5) for _ in range(2))
    grad = 0.5 + rng.random((r, c))
    grad[1, 4] = np.inf
    dy = _dev(grad, torch.bfloat16)
    dx, dgate, dup, ddown = _empty(r, p, torch.bfloat16), _empty(p, f, torch.bfloat16, ld=f + 3), _empty(p, f, torch.bfloat16, ld=f + 3), _empty(f, c, torch.bfloat16)
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_BF16, activation=B.BMGD_ACT_RELU) as block:
        block.backward(dy, x, gate, up, down, g, u, dx, dgate, dup, ddown)
    inf = lambda t: torch.isinf(t) & (t > 0)  # noqa: E731
    rows, cols = torch.arange(r, device="cuda") == 1, torch.arange(c, device="cuda") == 4
    assert inf(dx)[rows].all() and torch.isfinite(dx)[~rows].all()
    assert inf(dgate).all() and inf(dup).all()
    assert inf(ddown)[:, cols].all() and torch.isfinite(ddown)[:, ~cols].all()
    for t in (dgate, dup):                                     # nothing between the rows is written
        between = torch.as_strided(t, (p - 1, 3), (f + 3, 1), f)
        assert (between == 7).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("r,p,f,c", [(1, 512, 1000, 136), (17, 328, 240, 640), (40, 104, 200, 96), (134, 696, 136, 160), (300, 72, 64, 200), (700, 1024, 512, 264)])
def test_operands_at_odd_addresses_give_the_same_bits(r, p, f, c, kind):
    """Rows that begin anywhere come another way to the same sums in the same order."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    results = []
    for extra, offset in ((0, 0), (3, 1), (8, 3)):
        x, gate, up, down = _data(r, p, f, c, dtype, seed=r, lds=(p + extra, f + extra, f + extra, c + extra), offset=offset)
        dy = _dev(np.random.default_rng(r).standard_normal((r, c)), dtype, ld=c + extra, offset=offset)
        y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
        out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
        with B.GatedBlock(p, f, c, r, dtype=code) as block:
            block.forward(x, gate, up, down, y, g, u)
            block.backward(dy, x, gate, up, down, g, u, *out)
        results.append((y, g, u, *out))
    for other in results[1:]:
        for name, a, b in zip(("y", "g", "u", "dx", "dgate", "dup", "ddown"), results[0], other):
            assert torch.equal(a, b), name


@pytest.mark.parametrize("r", [1, 3, 20, 70, 200])
@pytest.mark.parametrize("p,f,c", [(8, 9, 10), (11, 12, 13), (14, 15, 17), (9, 65, 127), (71, 63, 9), (8, 8, 9), (7, 100, 100), (100, 100, 7), (100, 7, 100), (129, 130, 131)])
def test_widths_about_a_piece_and_a_step(r, p, f, c):
    import torch
    import paper_2312_08728_amd as B
    x, gate, up, down = _data(r, p, f, c, torch.bfloat16, seed=p + f)
    with B.GatedBlock(p, f, c, r, dtype=B.BMGD_BF16, activation=B.BMGD_ACT_SILU) as block:
        y, g, u = _empty(r, c, torch.bfloat16), _empty(r, f, torch.bfloat16), _empty(r, f, torch.bfloat16)
        block.forward(x, gate, up, down, y, g, u)
        _check_forward("bf16", "silu", x, gate, up, down, y, g, u)
        dy = _dev(np.random.default_rng(r).standard_normal((r, c)), torch.bfloat16)
        out = _empty(r, p, torch.bfloat16), _empty(p, f, torch.bfloat16), _empty(p, f, torch.bfloat16), _empty(f, c, torch.bfloat16)
        block.backward(dy, x, gate, up, down, g, u, *out)
        _check_backward("bf16", "silu", dy, x, gate, up, down, g, u, *out)
        for t in (y, g, u, *out):                              # nothing behind the last row is written
            assert (t.as_strided((8,), (1,), t.storage_offset() + t.numel()) == 7).all()
