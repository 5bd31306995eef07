"""Norm, 8-bit product and log probabilities at the ends of what is allowed: numbers as large and small as the header says, more rows than a launch has.

Tolerances are those of the operators' own tests.
"""
import numpy as np
import pytest

import test_gpu_int8 as I
import test_gpu_logprobs as L
import test_gpu_norm as N
from oracle import operators as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n", [100, 1500, 40_000])
@pytest.mark.parametrize("size,weight", [(2.0 ** -62, 1.0), (2.0 ** -40, 2.0 ** -20), (2.0 ** -40, 2.0 ** 100), (2.0 ** 50, 2.0 ** 70), (2.0 ** 50, 2.0 ** -30)])
def test_norm_of_large_and_small_rows(kind, n, size, weight):
    """Elements' sizes are within a factor of 8 of `size`, the weight's of `weight`; eps 0."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = N._types()[kind]
    gen = torch.Generator().manual_seed(n)
    sign = lambda *s: torch.randint(0, 2, s, generator=gen) * 2.0 - 1.0  # noqa: E731
    x = ((1 + 7 * torch.rand(3, n, generator=gen)) * sign(3, n) * size).to(dtype).cuda()
    w = ((1 + 3 * torch.rand(n, generator=gen)) * sign(n) * weight).to(dtype).cuda()
    y, c = torch.empty_like(x), torch.empty(3, n, dtype=torch.int8, device="cuda")
    scales, rstd = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    op = B.RMSNorm(n, dtype=code, eps=0.0)
    op.forward(x, w, y=y, codes=c, scales=scales, rstd=rstd)
    x64, w64 = N._np(x), N._np(w)
    y64, r64 = O.norm(x64, w64, 0.0)
    rel = (N._chain(n) + 8) * 2.0 ** -24
    assert (np.abs(N._np(rstd) - r64) <= r64 * rel).all()
    assert (np.abs(N._np(y) - y64) <= np.abs(y64) * (N.HALF[kind] + rel) + N.TINY[kind]).all()
    codes, top = O.codes_of(x64 * w64)
    assert (c.cpu().numpy() == codes).all()
    assert (np.abs(N._np(scales) - top * r64 / 127.0) <= top * r64 / 127.0 * rel).all()
    if weight != 1.0:
        return
    dy, dx, dw = torch.randn(3, n, generator=gen).to(dtype).cuda(), torch.empty_like(x), torch.empty_like(w)
    op.backward(dy, x, w, rstd, dx, dweight=dw)
    dy64, r64 = N._np(dy), N._np(rstd)
    dx64, dw64 = O.norm_backward(dy64, x64, w64, r64)
    wide = r64[:, None] * (np.abs(w64 * dy64) + np.abs(x64) * (r64 * r64 * np.abs(w64 * dy64 * x64).mean(1))[:, None])
    assert (np.abs(N._np(dx) - dx64) <= np.abs(dx64) * N.HALF[kind] + wide * (N._chain(n) + 10) * 2.0 ** -24).all()
    wide = (np.abs(dy64 * x64) * r64[:, None]).sum(0)
    assert (np.abs(N._np(dw) - dw64) <= np.abs(dw64) * N.HALF[kind] + wide * 40 * 2.0 ** -24).all()


@pytest.mark.parametrize("classes,rows", [(3, (1 << 22) + 9), (2049, (1 << 20) + 3)])
def test_scores_of_more_rows_than_a_launch_has(classes, rows):
    """Rows are looked at at both ends and around the borders of launches; the others by their sum: gradients of a row add up to nothing."""
    import torch
    import paper_2312_08728_amd as B
    x = torch.randn(rows, classes, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    labels = torch.arange(rows, device="cuda", dtype=torch.int32) % classes
    lp, h, kept = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda"), torch.empty(rows, 3, device="cuda")
    best, best_lp = torch.empty(rows, 2, dtype=torch.int32, device="cuda"), torch.empty(rows, 2, device="cuda")
    op = B.LogProbs(classes, top=2)
    op.forward(x, labels=labels, logprob=lp, entropy=h, kept=kept, top_classes=best, top_logprobs=best_lp)
    d = torch.full_like(x, 9.0)
    op.backward(x, kept, d, labels=labels, dlogprob=torch.ones(rows, device="cuda"))
    border = 1 << 21
    at = torch.tensor(sorted({i for i in (0, 1, 2, 3, 4, 5, border - 1, border, border + 1, (1 << 20) - 1, 1 << 20, rows - 3, rows - 2, rows - 1) if i < rows}), device="cuda")
    x64, chosen = L._np(x[at]), labels[at].cpu().numpy()
    logp, entropy = O.log_probabilities(x64)
    k = L._sum_error(classes)
    want = logp[np.arange(len(chosen)), chosen]
    L._close(lp[at], want, L.E * (2 * np.abs(want) + k))
    L._close(h[at], entropy, L.E * (k + 16) * (1 + np.log(classes + 1)))
    assert (best[at].cpu().numpy() == O.best(x64, 2)).all()
    want = O.logits_gradient(x64, chosen, np.ones(len(chosen)), np.zeros(len(chosen)))
    assert (np.abs(L._np(d[at]) - want) <= np.abs(want) * 2.0 ** -8 + L.E * (2 * np.abs(logp) + 2 * k) * 2 + L.TINY["bf16"]).all()
    # elements are off by half a step, 2^-8 of a row whose sizes add up to at most 2
    assert all(float(part.float().sum(1).abs().max()) <= 2 * 2.0 ** -8 + 1e-4 for part in d.split(1 << 18))
    assert float(lp.max()) <= 0 and float(h.max()) <= np.log(classes) * (1 + 1e-5)


def test_product_of_more_rows_than_a_launch_of_rows_has():
    import torch
    import paper_2312_08728_amd as B
    rows, p, out = (1 << 21) + 5, 16, 8
    x, w = I._codes(rows, p, 0, 0, 1), I._codes(out, p, 0, 0, 2)
    sx, sw = I._scales(rows, 3), I._scales(out, 4)
    y = torch.empty(rows, out, dtype=torch.bfloat16, device="cuda")
    B.Int8Product(p, out).forward(x, sx, w, sw, y)
    assert torch.equal(y.cpu(), I._want(x, sx, w, sw, torch.bfloat16))
    out32 = torch.empty(rows, p, device="cuda")
    B.RMSNorm(p).values(x, sx, out32)
    assert torch.equal(out32, sx[:, None] * x.float())
