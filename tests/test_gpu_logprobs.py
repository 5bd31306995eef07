"""Log probabilities, entropy, most probable classes and their gradient against 64-bit forms.

Tolerances count roundings of 2^-24.  With d = ln p, K additions of a lane (of at most ceil(classes / 64), and 30 over lanes, wavefronts and parts), and each e^(x - m) off
by the rounding of its exponent (2 |x - m| of them) and of the exponential itself (2): e^-t t is at most 1, so over a row these are at most 3 ln(classes) + 8.
"""
import math

import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -125, "f16": 2.0 ** -25, "f32": 2.0 ** -125}


def _types():
    import torch
    import paper_2312_08728_amd as B
    return {"bf16": (torch.bfloat16, B.BMGD_BF16), "f16": (torch.float16, B.BMGD_F16), "f32": (torch.float32, B.BMGD_F32)}


def _np(t):
    return t.double().cpu().numpy()


def _logits(rows, classes, dtype, pad=0, shift=0, seed=0, scale=2.5):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((rows * (classes + pad) + shift,), 7.0, dtype=dtype, device="cuda")
    m = flat[shift:].view(rows, classes + pad)[:, :classes]
    m.copy_(torch.randn(rows, classes, generator=gen, device="cuda") * scale)
    return m, flat


def _sum_error(classes):
    return -(-classes // 64) + 30 + 3 * math.log(classes + 1) + 8


def _forward(kind, x, labels, top):
    import torch
    import paper_2312_08728_amd as B
    rows, classes = x.shape
    new = lambda *s, dtype=torch.float32: torch.full(s, 77, dtype=dtype, device="cuda")  # noqa: E731
    out = dict(logprob=new(rows), entropy=new(rows), kept=new(rows, 3), top_classes=new(rows, top, dtype=torch.int32), top_logprobs=new(rows, top))
    op = B.LogProbs(classes, dtype=_types()[kind][1], top=top)
    op.forward(x, labels=labels, **out)
    return op, out


def _close(got, want, tolerance):
    got = _np(got)
    with np.errstate(invalid="ignore"):
        same = (got == want) | (np.isnan(got) & np.isnan(want)) | (np.abs(got - want) <= tolerance)
    assert same.all(), (got[~same][:5], want[~same][:5])


def _check(kind, x, labels, top):
    import torch
    rows, classes = x.shape
    op, out = _forward(kind, x, torch.from_numpy(labels).int().cuda(), top)
    x64 = _np(x)
    logp, entropy = O.log_probabilities(x64)
    k = _sum_error(classes)
    inside = (labels >= 0) & (labels < classes)
    chosen = np.where(inside, logp[np.arange(rows), np.clip(labels, 0, classes - 1)], np.where(labels < 0, 0.0, np.nan))
    finite = np.where(np.isfinite(chosen), chosen, 0.0)
    _close(out["logprob"], chosen, E * (2 * np.abs(finite) + k))
    _close(out["entropy"], entropy, E * (k + 16) * (1 + math.log(classes + 1)))
    if top:
        want = O.best(x64, top)
        assert (out["top_classes"].cpu().numpy() == want).all()
        want = np.take_along_axis(logp, want, 1)
        _close(out["top_logprobs"], want, E * (2 * np.abs(np.where(np.isfinite(want), want, 0.0)) + k))
    return op, out, x64, logp, entropy


def _gradient(kind, op, out, x, x64, labels, logp, entropy, into=None, dl=True, dh=True):
    import torch
    rows, classes = x.shape
    gen = torch.Generator().manual_seed(9)
    a, b = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    d = torch.full_like(x, 5.0) if into is None else into
    op.backward(x, out["kept"], d, labels=torch.from_numpy(labels).int().cuda() if dl else None, dlogprob=a.cuda() if dl else None, dentropy=b.cuda() if dh else None)
    a, b = a.double().numpy() if dl else np.zeros(rows), b.double().numpy() if dh else np.zeros(rows)
    want = O.logits_gradient(x64, labels if dl else np.full(rows, -1), a, b)
    lp = np.where(np.isfinite(logp), np.abs(logp), 0.0)
    p = np.where(np.isfinite(logp), np.exp(np.where(np.isfinite(logp), logp, 0.0)), 0.0)
    h = np.where(np.isfinite(entropy), entropy, 0.0)[:, None]
    wide = p * (np.abs(a)[:, None] + np.abs(b)[:, None] * (lp + h + 1.0))
    size = wide * (2 * lp + _sum_error(classes) + 16) * 2
    here = (labels >= 0) & (labels < classes)
    size[np.arange(rows)[here], labels[here]] += 2 * np.abs(a[here])
    _close(d, want, np.abs(np.where(np.isfinite(want), want, 0.0)) * HALF[kind] + E * size + TINY[kind])
    return d


def _labels(rows, classes, seed=0):
    rng = np.random.default_rng(seed)
    labels = rng.integers(0, classes, rows)
    labels[::7] = -1 - rng.integers(0, 100, len(labels[::7]))
    return labels


SIZES = [(1, 1), (3, 2), (5, 7), (4, 8), (6, 9), (2, 64), (9, 130), (5, 513), (70, 1000), (3, 2048), (3, 2049), (5, 4097), (2, 10_001), (40, 16_385), (3, 32_768), (2, 33_001), (1, 100_003),
         (2, 262_147), (600, 20_000)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,classes", SIZES)
def test_forward_and_gradient(kind, rows, classes):
    x, flat = _logits(rows, classes, _types()[kind][0], pad=classes % 3, shift=classes % 5, seed=rows)
    labels = _labels(rows, classes)
    if rows > 2:
        labels[2] = classes
    op, out, x64, logp, entropy = _check(kind, x, labels, min(5, classes))
    d = _gradient(kind, op, out, x, x64, labels, logp, entropy)
    import torch
    for dl, dh in ((True, False), (False, True)):
        _gradient(kind, op, out, x, x64, labels, logp, entropy, dl=dl, dh=dh)
    before = flat.clone()
    _gradient(kind, op, out, x, x64, labels, logp, entropy, into=x)              # in place
    assert torch.equal(x.nan_to_num(), d.nan_to_num())
    x.fill_(1.0)
    before.as_strided(x.shape, x.stride(), x.storage_offset()).fill_(1.0)
    assert torch.equal(flat, before)                                            # nothing between the rows is touched


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("top", [0, 1, 2, 17, 63, 64])
@pytest.mark.parametrize("rows,classes", [(3, 64), (2, 70), (5, 511), (3, 700), (2, 3000), (3, 20_000), (2, 50_001), (1, 300_000)])
def test_most_probable_classes(kind, top, rows, classes):
    x, _ = _logits(rows, classes, _types()[kind][0], shift=1, seed=top)
    _check(kind, x, _labels(rows, classes), top)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("top", [17, 33, 64])
@pytest.mark.parametrize("classes", [130, 655, 662, 1318, 1333])
def test_most_probable_classes_of_many_short_rows(kind, top, classes):
    """So many rows that each is a wavefront's: lists that are shortened first, pieces that just fit."""
    x, _ = _logits(1100, classes, _types()[kind][0], pad=classes % 3, shift=classes % 4, seed=classes + top)
    _check(kind, x, _labels(1100, classes), top)


def _rows_of_trouble(classes, dtype):
    """Rows by name, each with its own difficulty."""
    import torch
    low = torch.finfo(dtype).min
    up = torch.arange(classes, dtype=torch.float64)
    inf, nan = float("inf"), float("nan")
    base = torch.randn(classes, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    rows = {
        "equal": torch.zeros(classes), "no class": torch.full((classes,), -inf), "all lowest": torch.full((classes,), low), "rising": up / classes * 8, "falling": -up / classes * 8,
        "two values": (up % 2), "signed zeros": torch.where(up % 3 == 0, -0.0, 0.0), "one class": torch.full((classes,), -inf), "lowest but one": torch.full((classes,), low),
        "infinity": base.clone(), "nan": base.clone(), "many nan": torch.where(up % 2 == 1, nan, base), "both": base.clone(), "large": base * 0 + float(torch.finfo(dtype).max) / 2,
        "last is best": base.clone(), "far apart": base * 1e4, "one lane": torch.where(up % 4096 < 8, base + 100.0, base), "half masked": torch.where(up < classes // 2, base, -inf),
    }
    rows["one class"][classes - 1] = -3.0
    rows["lowest but one"][classes // 2] = 1.0
    rows["infinity"][classes // 3] = inf
    rows["nan"][classes // 2] = nan
    rows["both"][0], rows["both"][classes - 1] = inf, nan
    rows["last is best"][classes - 1] = 50.0
    return list(rows), torch.stack([r.double() for r in rows.values()]).to(dtype)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("classes", [3, 40, 1000, 9000, 40_000, 150_000])
@pytest.mark.parametrize("top", [0, 3, 64])
def test_rows_of_trouble(kind, classes, top):
    names, x = _rows_of_trouble(classes, _types()[kind][0])
    x = x.cuda()
    labels = np.arange(len(names)) % classes
    top = min(top, classes)
    op, out, x64, logp, entropy = _check(kind, x, labels, top)
    _gradient(kind, op, out, x, x64, labels, logp, entropy)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("classes,top", [(600, 64), (600, 33), (1300, 20), (1300, 64), (5000, 17), (20_000, 20), (20_000, 64), (90_000, 33)])
def test_equal_logits(kind, classes, top):
    """As many rows as one launch has workgroups for: equal in all classes, in a few values, in all but some, masked but for some."""
    import torch
    x = torch.zeros(600, classes)
    x[150:300] = torch.randint(0, 3, (150, classes), generator=torch.Generator().manual_seed(0)).float()
    x[300:] = -math.inf
    allowed = torch.randint(0, classes, (300, 10), generator=torch.Generator().manual_seed(1))
    x[300:].scatter_(1, allowed, 1.5)
    x[450:] = torch.where(x[450:] > 0, x[450:], torch.zeros(()))
    x = x.to(_types()[kind][0]).cuda()
    _check(kind, x[::50], np.zeros(12, dtype=np.int64), top)              # (rows far apart)
    _, out = _forward(kind, x, torch.zeros(600, dtype=torch.int32, device="cuda"), top)
    assert (out["top_classes"][::50].cpu().numpy() == O.best(_np(x[::50]), top)).all() and (out["top_classes"][:150] == torch.arange(top, device="cuda")).all()


def test_results_alone():
    """Each result by itself has the bits that it has with the others; no labels are needed without logprob."""
    import torch
    import paper_2312_08728_amd as B
    for rows, classes in ((3, 900), (2, 40_000)):
        x, _ = _logits(rows, classes, torch.float32, seed=3)
        labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
        _, out = _forward("f32", x, labels, 5)
        op = B.LogProbs(classes, dtype=B.BMGD_F32)
        for name in ("logprob", "entropy", "kept"):
            alone = torch.empty_like(out[name])
            op.forward(x, labels=labels if name == "logprob" else None, **{name: alone})
            assert torch.equal(alone, out[name])


def test_gradient_against_differences():
    import torch
    import paper_2312_08728_amd as B
    rows, classes, h = 2, 12, 2.0 ** -7
    x = torch.randn(rows, classes, generator=torch.Generator().manual_seed(0))
    labels = torch.tensor([3, 11], dtype=torch.int32, device="cuda")
    a, b = torch.tensor([1.0, -0.5]), torch.tensor([0.25, 1.5])
    op = B.LogProbs(classes, dtype=B.BMGD_F32)
    lp, en, kept = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 3, device="cuda")

    def value():
        op.forward(x.cuda(), labels=labels, logprob=lp, entropy=en, kept=kept)
        return float((lp.cpu().double() * a).sum() + (en.cpu().double() * b).sum())
    value()
    d = torch.empty(rows, classes, device="cuda")
    op.backward(x.cuda(), kept, d, labels=labels, dlogprob=a.cuda(), dentropy=b.cuda())
    # four values are off by 60 x 4 roundings at most; third derivatives of ln p and H are below 4
    tolerance = 4 * 240 * E / h + 8 * h * h / 6
    for i in np.ndindex(rows, classes):
        keep = float(x[i])
        x[i] = keep + h
        up = value()
        x[i] = keep - h
        down = value()
        x[i] = keep
        assert abs((up - down) / (2 * h) - float(d[i])) <= tolerance


@pytest.mark.parametrize("rows,classes", [(40, 900), (2, 60_000)])
def test_captured_and_replayed(rows, classes):
    """A step in a graph of torch's, with its workspace, replayed on other logits between eager calls; two graphs alive."""
    import torch
    import paper_2312_08728_amd as B
    op = B.LogProbs(classes, top=5)
    new = lambda: torch.randn(rows, classes, device="cuda").bfloat16()  # noqa: E731
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    g = torch.full((rows,), -1.0, device="cuda")

    def outputs():
        f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
        return dict(logprob=f(rows), entropy=f(rows), kept=f(rows, 3), top_classes=f(rows, 5).int(), top_logprobs=f(rows, 5)), torch.zeros(rows, classes, device="cuda").bfloat16()

    def step(x, out, d):
        op.forward(x, labels=labels, **out)
        op.backward(x, out["kept"], d, labels=labels, dlogprob=g, dentropy=g)
    made = []
    for _ in range(2):
        x, (out, d) = new(), outputs()
        step(x, out, d)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(x, out, d)
        made.append((graph, x, out, d))
    for _ in range(3):
        for _, x, _, _ in made:
            x.copy_(new())
        for graph, *_ in made:
            graph.replay()
        for _, x, out, d in made:
            out2, d2 = outputs()
            step(x, out2, d2)
            torch.cuda.synchronize()
            assert torch.equal(d, d2) and all(torch.equal(out[k], out2[k]) for k in out)


def test_rows_beyond_32_bits():
    import torch
    import paper_2312_08728_amd as B
    rows, classes, stride = 70, 100, 1 << 26
    x = torch.zeros((rows - 1) * stride + classes, dtype=torch.bfloat16, device="cuda").as_strided((rows, classes), (stride, 1))
    x[-1, 5] = 9.0
    op, out = _forward("bf16", x, torch.full((rows,), 5, dtype=torch.int32, device="cuda"), 2)
    assert out["top_classes"][-1].tolist() == [5, 0] and out["top_classes"][0].tolist() == [0, 1]
    op.backward(x, out["kept"], x, labels=torch.full((rows,), 5, dtype=torch.int32, device="cuda"), dlogprob=torch.ones(rows, device="cuda"))
    want = O.logits_gradient(np.where(np.arange(classes) == 5, 9.0, 0.0)[None], np.array([5]), np.ones(1), np.zeros(1))
    assert np.abs(_np(x[-1:]) - want).max() <= 2.0 ** -8
    assert abs(float(x[0, 0]) + 0.01) <= 0.01 * 2.0 ** -7


def test_no_rows_and_refusals():
    import torch
    import paper_2312_08728_amd as B
    op = B.LogProbs(32, top=2)
    x, f, i = torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    tc, tl = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    op.forward(x[:0], top_classes=tc[:0], top_logprobs=tl[:0])
    op.backward(x[:0], torch.zeros(0, 3, device="cuda"), x[:0])
    good = dict(top_classes=tc, top_logprobs=tl)
    for kw in (dict(), dict(top_classes=tc), dict(good, logprob=f), dict(good, labels=i.long(), logprob=f), dict(good, kept=f), dict(top_classes=tc.long(), top_logprobs=tl), dict(good, entropy=f.half()),
               dict(good, labels=i[:3], logprob=f), dict(good, entropy=f.cpu()), dict(good, logprob=f, entropy=f, labels=i)):
        with pytest.raises((ValueError, B.BmgdError)):
            op.forward(x, **kw)
    kept = torch.zeros(4, 3, device="cuda")
    for args, kw in (((x.float(), kept, x), {}), ((x, kept[:, :2], x), {}), ((x, kept, x[:3]), {}), ((x, kept, x), dict(dlogprob=f)), ((x, None, x), {})):
        with pytest.raises((ValueError, B.BmgdError)):
            op.backward(*args, **kw)
    wide = B.LogProbs(1 << 18)
    y = torch.zeros(1, 1 << 18, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.BmgdError, match="workspace"):
        wide.forward(y, entropy=f[:1], workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
