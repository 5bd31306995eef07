"""8-bit product and the layout of its weights.  Integer sums are exact and the roundings behind them are named, so results are compared bit by bit."""
import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu


def _types():
    import torch
    import paper_2312_08728_amd as B
    return {"bf16": (torch.bfloat16, B.BMGD_BF16), "f16": (torch.float16, B.BMGD_F16), "f32": (torch.float32, B.BMGD_F32)}


def _codes(rows, n, pad, shift, seed, low=-127):
    import torch
    gen = torch.Generator().manual_seed(seed)
    flat = torch.randint(low, 128, (rows * (n + pad) + shift + 64,), generator=gen, dtype=torch.int8).cuda()
    return flat[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n]


def _scales(n, seed):
    import torch
    return (torch.rand(n, generator=torch.Generator().manual_seed(seed)) * 1e-2 + 1e-4).cuda()


def _want(x, sx, w, sw, dtype):
    import torch
    total = x.cpu().double() @ w.cpu().double().t()                      # (exact: below 2^53)
    return (total.float() * sx.cpu()[:, None] * sw.cpu()).to(dtype)


def _check(rows, p, out, kind, pads=(0, 0, 0), shifts=(0, 0), low=-127):
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    x, w = _codes(rows, p, pads[0], shifts[0], 1, low), _codes(out, p, pads[1], shifts[1], 2, low)
    sx, sw = _scales(rows, 3), _scales(out, 4)
    flat = torch.full((rows * (out + pads[2]) + 3,), 3.0, dtype=dtype, device="cuda")
    y = flat[1:1 + rows * (out + pads[2])].view(rows, out + pads[2])[:, :out]
    y.fill_(9)
    others = int((flat == 3).sum())
    B.Int8Product(p, out, dtype=code).forward(x, sx, w, sw, y)
    assert torch.equal(y.cpu(), _want(x, sx, w, sw, dtype))
    y.fill_(9)
    assert int((flat == 3).sum()) == others


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows", [1, 2, 16, 17, 32, 33, 64, 65, 100])
@pytest.mark.parametrize("p,out", [(1, 1), (5, 3), (15, 20), (16, 16), (17, 33), (63, 65), (64, 64), (100, 37), (130, 129), (512, 100), (1365, 70), (4096, 48), (4111, 17)])
def test_few_rows(kind, rows, p, out):
    _check(rows, p, out, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,p,out", [(300, 256, 300), (257, 144, 513), (129, 1040, 1000), (1000, 128, 1500), (2049, 272, 2111), (4100, 512, 4097), (4096, 208, 4096), (8200, 64, 2056)])
def test_large(kind, rows, p, out):
    """Tiles of every kind with rows, columns and steps that end inside one."""
    _check(rows, p, out, kind)


@pytest.mark.parametrize("rows", [1, 20, 200, 2100])
@pytest.mark.parametrize("p,pads,shifts", [(77, (0, 0, 0), (0, 0)), (64, (1, 0, 1), (0, 0)), (64, (0, 3, 0), (0, 0)), (160, (0, 0, 3), (1, 0)), (160, (16, 0, 2), (0, 8)), (31, (1, 1, 1), (15, 1)),
                                           (1, (0, 0, 0), (0, 0)), (9, (2, 0, 5), (3, 4)), (16, (16, 32, 0), (16, 16))])
def test_operands_at_any_address(rows, p, pads, shifts):
    _check(rows, p, 150 if rows < 2000 else 2300, "f16", pads, shifts)


def test_largest_sums():
    """128^2 131071 is below 2^31: all codes -128, and the same against 127."""
    import torch
    import paper_2312_08728_amd as B
    p = 131_071
    one = torch.ones(40, device="cuda")
    for rows in (3, 40):
        x, w = torch.full((rows, p), -128, dtype=torch.int8, device="cuda"), torch.full((40, p), -128, dtype=torch.int8, device="cuda")
        w[1::2] = 127
        y = torch.empty(rows, 40, device="cuda")
        B.Int8Product(p, 40, dtype=B.BMGD_F32).forward(x, one[:rows], w, one, y)
        want = torch.where(torch.arange(40) % 2 == 0, 16384.0 * p, -128.0 * 127.0 * p).float()
        assert torch.equal(y.cpu(), want.expand(rows, 40))


def test_scales_that_are_zero_or_not_finite():
    import torch
    import paper_2312_08728_amd as B
    for rows in (4, 70):
        x, w = _codes(rows, 64, 0, 0, 1), _codes(24, 64, 0, 0, 2)
        sx, sw = torch.ones(rows, device="cuda"), torch.ones(24, device="cuda")
        sx[1], sx[2], sw[3], sw[4] = 0.0, float("nan"), float("nan"), float("inf")
        y = torch.empty(rows, 24, device="cuda")
        B.Int8Product(64, 24, dtype=B.BMGD_F32).forward(x, sx, w, sw, y)
        want = _want(x, sx, w, sw, torch.float32)
        assert torch.equal(torch.isnan(y.cpu()), torch.isnan(want)) and torch.equal(torch.nan_to_num(y.cpu()), torch.nan_to_num(want))


def test_rows_beyond_32_bits():
    """Rows that lie so far apart that the last ones begin behind 2^32 elements, of operands and results."""
    import torch
    import paper_2312_08728_amd as B
    for rows, far in ((20, 1 << 28), (70, 1 << 26)):
        p, out = 64, 70
        x = torch.zeros((rows - 1) * far + p, dtype=torch.int8, device="cuda").as_strided((rows, p), (far, 1))
        w = torch.zeros((out - 1) * (1 << 26) + p, dtype=torch.int8, device="cuda").as_strided((out, p), (1 << 26, 1))
        y = torch.zeros((rows - 1) * far + out, dtype=torch.bfloat16, device="cuda").as_strided((rows, out), (far, 1))
        a, b = _codes(rows, p, 0, 0, 1), _codes(out, p, 0, 0, 2)
        x.copy_(a)
        w.copy_(b)
        sx, sw = _scales(rows, 3), _scales(out, 4)
        B.Int8Product(p, out).forward(x, sx, w, sw, y)
        assert torch.equal(y.cpu(), _want(a, sx, b, sw, torch.bfloat16))
        del x, w, y


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("p,out,pad", [(1, 1, 0), (7, 130, 1), (64, 64, 0), (100, 65, 2), (513, 200, 0), (2049, 96, 3)])
def test_layout_of_weights(kind, p, out, pad):
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()[kind]
    flat = torch.randn(p * (out + pad) + 1, generator=torch.Generator().manual_seed(0)).to(dtype)
    m = flat[1:].view(p, out + pad)[:, :out]
    special = out > 60
    if special:
        m[:, 3], m[:, 7] = 0, 0
        m[p // 2, 7] = 2.0 ** -119
        m[p - 1, 11], m[0, 20] = float("inf"), float("nan")
    m = flat.cuda()[1:].view(p, out + pad)[:, :out]
    w = torch.full((out, p + pad), 5, dtype=torch.int8, device="cuda")
    scales = torch.empty(out, device="cuda")
    B.Int8Product(p, out, dtype=code).quantize(m, w[:, :p], scales)
    codes, top = O.codes_of(m.double().cpu().numpy().T)
    assert (w[:, :p].cpu().numpy() == codes).all() and (w[:, p:] == 5).all()
    got, want = scales.cpu().numpy(), top.astype(np.float32) / np.float32(127)
    assert np.array_equal(got, want, equal_nan=True)


def test_no_rows_and_refusals():
    import torch
    import paper_2312_08728_amd as B
    op = B.Int8Product(32, 8)
    x, w, f = torch.zeros(4, 32, dtype=torch.int8, device="cuda"), torch.zeros(8, 32, dtype=torch.int8, device="cuda"), torch.zeros(8, device="cuda")
    y = torch.zeros(4, 8, dtype=torch.bfloat16, device="cuda")
    op.forward(x[:0], f[:0], w, f, y[:0])
    for args in ((x, f[:4], w, f, y.float()), (x, f, w, f, y), (x.float(), f[:4], w, f, y), (x, f[:4], w[:7], f, y), (x, f[:4], w.t().contiguous().t(), f, y), (x, f[:4], w, f.double(), y),
                 (x, f[:4], w, f, y.cpu()), (x, f[:4], w.cpu(), f, y), (x, f[:4], None, f, y)):
        with pytest.raises((ValueError, B.BmgdError)):
            op.forward(*args)
    for args in ((y, w, f), (torch.zeros(32, 8, dtype=torch.bfloat16, device="cuda"), w.t().contiguous(), f), (torch.zeros(32, 8, device="cuda"), w, f)):
        with pytest.raises(ValueError):
            op.quantize(*args)
    with pytest.raises(ValueError):
        op.values(x, f[:4], torch.zeros(4, 32, dtype=torch.int8, device="cuda"))
