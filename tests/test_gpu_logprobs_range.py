"""Log probabilities, entropy and gradient of logits of any size: ln p depends on differences of logits alone, whatever they lie around.

Tolerances as in test_gpu_logprobs, and four roundings more: an exponent is rounded with what the row's reference has lost of the largest logit's, at most 1 in size, so each
of exponent, sum, logarithm and difference is off by one rounding of a number that is larger by 1.
"""
import math

import numpy as np
import pytest

import test_gpu_logprobs as T

pytestmark = pytest.mark.gpu

BORDER = 2.0 ** 24
SIZES = [1.0e6, BORDER / 2, BORDER - 64, BORDER, BORDER + 64, 3.0e9, 1.0e10, 1.0e15, 1.0e20, 1.0e30, 5.0e36, 9.9e36, 1.1e37, 1.0e38]


@pytest.fixture(autouse=True)
def _four_roundings_more(monkeypatch):
    kept = T._sum_error
    monkeypatch.setattr(T, "_sum_error", lambda classes: kept(classes) + 4)


def _round(kind, x):
    import torch
    return torch.from_numpy(x).to(T._types()[kind][0])


def _both(kind, x, top):
    rows, classes = x.shape
    labels = T._labels(rows, classes)
    x = x.cuda()
    op, out, x64, logp, entropy = T._check(kind, x, labels, top)
    T._gradient(kind, op, out, x, x64, labels, logp, entropy)
    return out, logp, entropy


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("classes,top", [(3, 2), (1000, 5), (2500, 0), (9001, 5), (50_257, 9), (40_000, 0)])
def test_rows_of_any_size(kind, classes, top):
    """Equal logits (a row masked with a finite number), and logits on the type's steps around them, of both signs."""
    import torch
    rng = np.random.default_rng(classes)
    rows = []
    for size in SIZES:
        for v in (size, -size):
            step = float(torch.finfo(T._types()[kind][0]).eps) * size
            rows.append(np.full(classes, v))
            rows.append(v + step * rng.integers(-2, 3, classes))
            rows.append(np.where(rng.random(classes) < 0.5, v, -np.inf))
            rows.append(np.where(np.arange(classes) == classes - 1, 3.0, v))
    out, logp, entropy = _both(kind, _round(kind, np.stack(rows)), top)
    equal = out["entropy"][::4].double().cpu().numpy()
    assert np.abs(equal - math.log(classes)).max() <= 2.0 ** -24 * (T._sum_error(classes) + 16) * (1 + math.log(classes + 1))


@pytest.mark.parametrize("rows", [1, 3, 520])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("classes", [33, 2000, 9001, 50_257])
def test_logits_around_the_border(rows, sign, classes):
    """fp32, where a row's largest logit is on either side of 2^24, and its lanes', wavefronts' and parts' largest ones on both."""
    import torch
    if rows * classes > 10_000_000:
        rows = 40
    gen = torch.Generator().manual_seed(classes)
    x = sign * BORDER + torch.randint(-8, 9, (rows, classes), generator=gen) * 2.0
    # stretches of a row, as long as a part, a wavefront's or a lane's share, all on one side or far away
    for first, each in ((0, 8192), (1, 512), (2, 8)):
        side = (torch.arange(classes) // each) % 3
        part = x[first::3]
        x[first::3] = torch.where(side == 0, part, torch.where(side == 1, part - 24.0, part - 3000.0))
    _both("f32", x.float()[: min(rows, 40)], 5 if classes > 33 else 0)
    if rows > 40:
        labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
        _, out = T._forward("f32", x.float().cuda(), labels, 5)
        logp, entropy = T.O.log_probabilities(x.double().numpy()[::50])
        k = T._sum_error(classes)
        T._close(out["entropy"][::50], entropy, T.E * (k + 16) * (1 + math.log(classes + 1)))
        T._close(out["logprob"][::50], logp[:, 0], T.E * (2 * np.abs(logp[:, 0]) + k))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("fill", [-1.0e9, -1.0e10, -1.0e30, -3.0e38])
@pytest.mark.parametrize("classes", [1000, 9001, 50_257])
def test_masks_of_a_finite_number(kind, fill, classes):
    """Rows masked with a finite number: in all classes but some, whole parts of them, in all."""
    import torch
    x = torch.randn(4, classes, generator=torch.Generator().manual_seed(0)).double().numpy()
    x[0, 5:] = fill
    x[1, : classes - 3] = fill
    x[2, :] = fill
    x[3, classes // 4: classes // 2] = fill
    _both(kind, _round(kind, x), 5)


@pytest.mark.parametrize("classes", [5, 900, 9001, 50_257])
def test_what_is_kept(classes):
    """The largest logit, log2 of the sum of 2^(x log2 e - r) and the entropy, r = fl(largest log2 e) up to 2^24 and largest log2 e beyond: with r again it is the logarithm of
    the sum of e^x.  (log2 e as the kernels have it, 1.44269504f: off by less than 2^-25 of it, of every difference x - largest; they are below 80 here.)"""
    import torch
    shifts = np.array([0.0, 30.0, -1000.0, 1.0e6, -9.0e6, 2.0 ** 24 + 64, -1.0e9, 1.0e12])
    x = torch.randn(len(shifts), classes, generator=torch.Generator().manual_seed(2)) * 5
    x = (x.double() + torch.from_numpy(shifts)[:, None]).float()
    _, out = T._forward("f32", x.cuda(), torch.zeros(len(shifts), dtype=torch.int32, device="cuda"), 2)
    kept, x64 = out["kept"].cpu().numpy(), x.double().numpy()
    largest = x64.max(1)
    assert (kept[:, 0] == largest).all() and (kept[:, 2] == out["entropy"].cpu().numpy()).all()
    log2e = np.float32(1.44269504)
    lost = np.where(np.abs(largest) < BORDER, largest * float(log2e) - (kept[:, 0] * log2e).astype(np.float64), 0.0)
    want = np.log2(np.exp(x64 - largest[:, None]).sum(1)) + lost
    # the sum's roundings are relative, so log2 e of them in the logarithm, which is rounded to fp32 within two steps of a number below 32
    assert (np.abs(kept[:, 1] - want) <= 1.45 * T.E * T._sum_error(classes) + 80 * 1.45 * 2.0 ** -25 + 2 * 32 * 2.0 ** -23).all()
    assert (np.abs(lost[3:5]) > 1e-3).any()
