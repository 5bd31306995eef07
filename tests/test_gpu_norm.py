"""Root-mean-square norm, its gradient and its 8-bit codes against 64-bit forms.

Tolerances count roundings.  A result is rounded by at most half a step of its type, relative.  Sums in 32 bits: a chain of k additions is off by
at most k half steps of what is added up; a lane adds at most 8 ceil(n / 512) elements (16 ceil(n / 8192) where more wavefronts share a row, which is less),
then six steps over lanes and up to 16 over wavefronts; a few more roundings belong to the mean, its root and the products.
"""
import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -126, "f16": 2.0 ** -25, "f32": 2.0 ** -126}    # absolute, where numbers are no longer normal


def _types():
    import torch
    import paper_2312_08728_amd as B
    return {"bf16": (torch.bfloat16, B.BMGD_BF16), "f16": (torch.float16, B.BMGD_F16), "f32": (torch.float32, B.BMGD_F32)}


def _chain(n):
    return 8 * -(-n // 512) + 30


def _strided(rows, n, dtype, pad, scale=1.0, seed=0, shift=1):
    """Rows that lie pad elements apart, from an odd element on."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (n + pad) + shift + 8,), 3.0, dtype=dtype, device="cuda") if dtype.is_floating_point else torch.full((rows * (n + pad) + shift + 8,), 3, dtype=dtype, device="cuda")
    m = flat[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n]
    if dtype.is_floating_point:
        m.copy_(torch.randn(rows, n, generator=gen, device="cuda") * scale)
    return m, flat


def _np(t):
    return t.double().cpu().numpy()


SHAPES = [(1, 1, 0), (3, 7, 0), (5, 8, 3), (2, 129, 0), (9, 512, 0), (7, 513, 1), (6, 1024, 8), (3, 1365, 0), (4, 2048, 5), (2, 4096, 0), (3, 4097, 2), (2, 8192, 0),
          (2, 16_384, 0), (2, 16_385, 0), (2, 32_768, 1), (2, 32_769, 3), (1, 100_003, 0), (700, 40, 2)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,n,pad", SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_forward(kind, rows, n, pad, residual):
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    x, _ = _strided(rows, n, dtype, pad, seed=1)
    q = _strided(rows, n, dtype, pad + 1, seed=2, shift=0)[0] if residual else None
    w = (torch.randn(n, generator=torch.Generator().manual_seed(3)) + 1.0).to(dtype).cuda()
    (s, sflat), (y, yflat), (c, cflat) = _strided(rows, n, dtype, 3), _strided(rows, n, dtype, 5, shift=2), _strided(rows, n, torch.int8, 1)
    for t in (s, y, c):
        t.fill_(9)
    scales, rstd = torch.full((rows,), -1.0, device="cuda"), torch.full((rows,), -1.0, device="cuda")
    eps = 1e-5
    op = B.RMSNorm(n, dtype=code, eps=eps)
    op.forward(x, w, y=y, residual=q, sum=s, codes=c, scales=scales, rstd=rstd)
    want = (x.float() + q.float()).to(dtype) if residual else x
    assert torch.equal(s, want)
    s64, w64 = _np(want), _np(w)
    y64, r64 = O.norm(s64, w64, float(np.float32(eps)))
    rel = (_chain(n) + 8) * 2.0 ** -24
    assert (np.abs(_np(y) - y64) <= np.abs(y64) * (HALF[kind] + rel) + TINY[kind]).all()
    assert (np.abs(_np(rstd) - r64) <= r64 * rel).all()
    codes, top = O.codes_of(s64 * w64)
    assert (c.cpu().numpy() == codes).all()
    assert (np.abs(_np(scales) - top * r64 / 127.0) <= top * r64 / 127.0 * rel).all()
    for flat, m in ((sflat, s), (yflat, y), (cflat, c)):                 # nothing between the rows is touched
        assert int((flat == 3).sum()) >= flat.numel() - m.numel()
    # each on its own, without a weight, into the operand
    only, z = torch.empty_like(y), x.clone()
    op.forward(x, w, y=only, residual=q)
    assert torch.equal(only, y)
    c2, sc2 = torch.empty_like(c), torch.empty_like(scales)
    op.forward(x, w, codes=c2, scales=sc2, residual=q)
    assert torch.equal(c2, c) and torch.equal(sc2, scales)
    op.forward(z, y=z, residual=q)
    y64 = O.norm(s64, np.ones(n), float(np.float32(eps)))[0]
    assert (np.abs(_np(z) - y64) <= np.abs(y64) * (HALF[kind] + rel) + TINY[kind]).all()
    out = torch.empty(rows, n, device="cuda")
    op.values(c, scales, out)
    assert torch.equal(out, scales[:, None] * c.float())
    half = torch.empty(rows, n + 1, dtype=torch.bfloat16, device="cuda")[:, 1:]
    op.values(c, scales, half)
    assert torch.equal(half, out.bfloat16())


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n", [37, 1000, 4096, 40_000])
def test_sum_in_place(kind, n):
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    x, q = _strided(3, n, dtype, 0, seed=1)[0], _strided(3, n, dtype, 0, seed=2)[0]
    y, z = torch.empty(3, n, dtype=dtype, device="cuda"), torch.empty(3, n, dtype=dtype, device="cuda")
    want = (x.float() + q.float()).to(dtype)
    op = B.RMSNorm(n, dtype=code)
    op.forward(x, y=y, residual=q)
    for into in (x.clone(), q.clone()):
        a, b = (into, q) if torch.equal(into, x) else (x, into)
        op.forward(a, y=z, residual=b, sum=into)
        assert torch.equal(into, want) and torch.equal(z, y)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,n,pad", [(1, 1, 0), (3, 7, 2), (9, 512, 0), (130, 520, 1), (5, 1024, 0), (3, 1365, 0), (700, 2048, 0), (3, 4096, 3), (1100, 4104, 0), (2, 8192, 0), (600, 8000, 0),
                                        (2, 16_384, 1), (3, 16_390, 0), (2, 33_000, 0), (2100, 64, 0), (1024, 64, 0), (1024, 72, 3), (1023, 2048, 0), (65, 16_384, 0), (300, 8192, 0)])
@pytest.mark.parametrize("way", ["all", "plain"])
def test_backward(kind, rows, n, pad, way):
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    s, dy = _strided(rows, n, dtype, pad, seed=1)[0], _strided(rows, n, dtype, 1, seed=2, shift=2)[0]
    ds = _strided(rows, n, dtype, 2, seed=3)[0] if way == "all" else None
    w = (torch.randn(n, generator=torch.Generator().manual_seed(4)) + 1.0).to(dtype).cuda() if way == "all" else None
    dx, flat = _strided(rows, n, dtype, 3, seed=5)
    dw = torch.empty(n, dtype=dtype, device="cuda") if way == "all" else None
    op = B.RMSNorm(n, dtype=code)
    rstd = torch.empty(rows, device="cuda")
    op.forward(s, w, y=torch.empty_like(s), rstd=rstd)
    op.backward(dy, s, w, rstd, dx, dweight=dw, dsum=ds)
    s64, dy64, r64, w64 = _np(s), _np(dy), _np(rstd), _np(w) if w is not None else np.ones(n)
    ds64 = _np(ds) if ds is not None else np.zeros_like(s64)
    dx64, dw64 = O.norm_backward(dy64, s64, w64, r64, ds64)
    size = r64[:, None] * (np.abs(w64 * dy64) + np.abs(s64) * (r64 * r64 * np.abs(w64 * dy64 * s64).mean(1))[:, None]) + np.abs(ds64)
    assert (np.abs(_np(dx) - dx64) <= np.abs(dx64) * HALF[kind] + size * (_chain(n) + 10) * 2.0 ** -24 + TINY[kind]).all()
    assert int((flat == 3).sum()) >= flat.numel() - dx.numel()
    if way == "all":
        # a part has at most ceil(rows / 512) + 4 rows of a lane, 512 parts are added eight by eight by eight; or a thread has every 64th row of 1,024, 16 threads are added and then up to 16
        chain = max(-(-rows // 512) + 4 + 8 + 8 + 8, min(16, -(-rows // 64)) + 16 + 16) + 4
        size = (np.abs(dy64 * s64) * r64[:, None]).sum(0)
        assert (np.abs(_np(dw) - dw64) <= np.abs(dw64) * HALF[kind] + size * chain * 2.0 ** -24 + TINY[kind]).all()
        for into in (dy, ds):                                            # in place, always the same bits
            a, b, again = dy.clone(), ds.clone(), torch.empty_like(dw)
            to = a if into is dy else b
            op.backward(a, s, w, rstd, to, dweight=again, dsum=b)
            assert torch.equal(to, dx) and torch.equal(again, dw)
        none = torch.empty_like(dx)
        op.backward(dy, s, w, rstd, none, dsum=ds)
        assert torch.equal(none, dx)


def test_gradients_against_differences():
    """Of sum y g, in 32 bits: central differences of the kernel's own forward pass."""
    import torch
    import paper_2312_08728_amd as B
    rows, n, h = 2, 24, 2.0 ** -8
    gen = torch.Generator().manual_seed(0)
    s, w, g = (torch.randn(*shape, generator=gen) for shape in ((rows, n), (n,), (rows, n)))
    op = B.RMSNorm(n, dtype=B.BMGD_F32)
    y, rstd = torch.empty(rows, n, device="cuda"), torch.empty(rows, device="cuda")

    def value(a, b):
        op.forward(a.cuda(), b.cuda(), y=y, rstd=rstd)
        return float((y.cpu().double() * g.double()).sum())
    value(s, w)
    dx, dw = torch.empty(rows, n, device="cuda"), torch.empty(n, device="cuda")
    op.backward(g.cuda(), s.cuda(), w.cuda(), rstd, dx, dweight=dw)
    # values of about 10 are off by 48 x 40 x 2^-24 at most, third derivatives here stay below 50
    tolerance = 48 * 40 * 2.0 ** -24 / h + 50 * h * h / 6
    for t, d in ((s, dx.cpu()), (w, dw.cpu())):
        for i in np.ndindex(*t.shape):
            keep = float(t[i])
            t[i] = keep + h
            up = value(s, w)
            t[i] = keep - h
            down = value(s, w)
            t[i] = keep
            assert abs((up - down) / (2 * h) - float(d[i])) <= tolerance


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n", [20, 3000, 40_000])
def test_rows_that_are_zero_tiny_or_not_finite(kind, n):
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    x = torch.randn(6, n, generator=torch.Generator().manual_seed(0)).to(dtype)
    x[0] = 0
    x[1] = 0
    x[1, n // 2] = 2.0 ** -119                    # (f16: zero)
    x[2, n - 1] = float("inf")
    x[3, 0] = float("nan")
    w = torch.ones(n, dtype=dtype)
    op = B.RMSNorm(n, dtype=code)
    y, c, scales = torch.empty(6, n, dtype=dtype, device="cuda"), torch.full((6, n), 5, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    op.forward(x.cuda(), w.cuda(), y=y, codes=c, scales=scales)
    assert not y[0].any() and not c[:4].any() and not scales[:2].any() and torch.isnan(scales[2:4]).all()
    assert torch.isnan(y[2, n - 1]) and torch.isnan(y[3]).all() and torch.isfinite(y[4:].float()).all()
    out = torch.empty(6, n, device="cuda")
    op.values(c, scales, out)
    assert not out[:2].any() and torch.isnan(out[2:4]).all() and torch.isfinite(out[4:]).all()
    # a weight that is not finite
    w[1] = float("-inf")
    op.forward(x.cuda(), w.cuda(), codes=c, scales=scales)
    assert torch.isnan(scales[4:]).all() and not c[4:].any()


def test_no_rows():
    import torch
    import paper_2312_08728_amd as B
    op = B.RMSNorm(70)
    x, none = torch.empty(0, 70, dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda")
    dw = torch.ones(70, dtype=torch.bfloat16, device="cuda")
    op.forward(x, y=x.clone(), rstd=none)
    op.backward(x, x.clone(), None, none, x.clone(), dweight=dw)
    assert not dw.any()
    op.values(torch.empty(0, 70, dtype=torch.int8, device="cuda"), none, x.clone())


def test_rows_beyond_32_bits_and_many_rows():
    """The last row begins behind 2^32 elements; more rows than a launch has."""
    import torch
    import paper_2312_08728_amd as B
    n, stride = 64, 1 << 20
    rows = (1 << 12) + 3
    flat = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda")
    x = flat.view(rows, stride)[:, 5:5 + n]
    x[-1] = torch.arange(n, device="cuda").bfloat16()
    x[-2] = 1.0
    y = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    op = B.RMSNorm(n, eps=0.5)
    op.forward(x, y=x.clone(), sum=y)
    op.forward(x, y=x)
    assert torch.equal(x[-2].float(), torch.full((n,), 1.0 / 1.5 ** 0.5, device="cuda").bfloat16().float())
    assert torch.equal(y[-1], torch.arange(n, device="cuda").bfloat16()) and not x[:-2].any()
    del flat, x
    rows = (1 << 21) + 5
    x = torch.ones(rows, 8, dtype=torch.bfloat16, device="cuda")
    x[-1] = 2.0
    y = torch.zeros_like(x)
    B.RMSNorm(8, eps=0.0).forward(x, y=y)
    assert (y == 1.0).all()


@pytest.mark.parametrize("n,rows", [(40, 300), (41, 300), (5000, 900), (4096, 1100)])
def test_a_training_step_in_a_graph(n, rows):
    """Forward and backward with the weight's gradient, captured and replayed on other inputs, eager calls in between."""
    import torch
    import paper_2312_08728_amd as B
    op = B.RMSNorm(n)
    new = lambda: torch.randn(rows, n, device="cuda").bfloat16()  # noqa: E731
    x, dy, w = new(), new(), torch.randn(n, device="cuda").bfloat16()
    y, dx, dw, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty(rows, device="cuda")

    def step(x, dy, w, y, dx, dw, rstd):
        op.forward(x, w, y=y, rstd=rstd)
        op.backward(dy, x, w, rstd, dx, dweight=dw)
    step(x, dy, w, y, dx, dw, rstd)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x, dy, w, y, dx, dw, rstd)
    for _ in range(4):
        x.copy_(new())
        dy.copy_(new())
        graph.replay()
        eager = [torch.empty_like(t) for t in (y, dx, dw, rstd)]
        step(x, dy, w, *eager)
        torch.cuda.synchronize()
        for a, b in zip((y, dx, dw, rstd), eager):
            assert torch.equal(a, b)


def test_refusals():
    import torch
    import paper_2312_08728_amd as B
    op = B.RMSNorm(16)
    x, f = torch.zeros(4, 16, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, device="cuda")
    bad = [dict(y=x.float()), dict(y=x[:3]), dict(y=x.t().contiguous().t()), dict(y=x, weight=f), dict(codes=x), dict(y=x.cpu()), dict(y="y")]
    for kw in bad:
        with pytest.raises(ValueError):
            op.forward(x.clone(), **kw)
    for kw in (dict(), dict(sum=x), dict(codes=torch.zeros(4, 16, dtype=torch.int8, device="cuda")), dict(y=x, sum=x)):
        with pytest.raises(B.BmgdError):
            op.forward(x.clone(), **kw)
    for args in ((x, x, None, f, x), (x, x.clone(), None, f[:3], x), (x, x.clone(), x[0], f.half(), x)):
        with pytest.raises((B.BmgdError, ValueError)):
            op.backward(*args)
    with pytest.raises(ValueError, match="workspace"):
        op.backward(x, x.clone(), None, f, x, dweight=x[0].clone(), workspace=torch.zeros(1 << 20))
    many, of_many = torch.zeros(5000, 16, dtype=torch.bfloat16, device="cuda"), torch.zeros(5000, device="cuda")
    with pytest.raises(B.BmgdError, match="workspace"):
        op.backward(many, many.clone(), None, of_many, many, dweight=x[0].clone(), workspace=torch.zeros(64, device="cuda"))
