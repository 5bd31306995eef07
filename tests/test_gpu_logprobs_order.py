"""The most probable classes where logits are equal across a row's parts, turns and ends: of equal ones the lowest class comes first, wherever the others lie.

Rows whose ends lie inside 16 bytes, with equal logits in that last piece and in the turn before it; larger ones at the row's beginning, in pieces of their own, so that
the last piece's number is the one that later ones have to reach.
"""
import numpy as np
import pytest

from oracle import operators as O
from test_gpu_logprobs import _check, _labels, _types

pytestmark = pytest.mark.gpu

# rows, classes: one wavefront to a row (many rows), four (few classes too many for one, or few rows), four over many turns, parts that are joined
SIZES = {"bf16": [(1100, 2500), (1100, 4001), (2, 9001), (520, 20_003), (3, 50_257)], "f16": [(1100, 2500), (1100, 4001), (2, 9001), (520, 20_003), (3, 50_257)],
         "f32": [(1100, 1301), (1100, 2047), (2, 9001), (520, 10_001), (3, 50_257)]}
CASES = [(kind, rows, classes) for kind in SIZES for rows, classes in SIZES[kind]]


def _patterns(classes, top, n, seed):
    """Rows (fp32) of zeros but for: `above` larger logits, one at the beginning of a piece each; one value at some of the last n classes and at some lower ones."""
    rng = np.random.default_rng(seed)
    rows = []
    for above in {0, top - 1, max(top - 2, 0)}:
        for lower in ([classes - 20], [classes // 2, classes - 9], [classes - 1 - n], []):
            for last in ([classes - 1], [classes - 2, classes - 1], [classes - 1 - int(rng.integers(n))]):
                x = np.zeros(classes, dtype=np.float32)
                x[8 * np.arange(1, above + 1)] = 9.0
                x[lower] = 5.0
                x[last] = 5.0
                rows.append(x)
    return np.stack(rows)


@pytest.mark.parametrize("kind,rows,classes", CASES)
@pytest.mark.parametrize("top", [1, 5, 16, 64])
def test_equal_logits_at_the_end_of_a_row(kind, rows, classes, top):
    import torch
    import paper_2312_08728_amd as B
    made = _patterns(classes, top, 8 if kind != "f32" else 4, seed=classes)
    want = torch.from_numpy(O.best(made.astype(np.float64), top))
    op = B.LogProbs(classes, dtype=_types()[kind][1], top=top)
    best, logprobs = torch.empty(rows, top, dtype=torch.int32, device="cuda"), torch.empty(rows, top, device="cuda")
    made = torch.from_numpy(made).to(_types()[kind][0]).cuda()
    for first in range(0, len(made), rows):                                    # (as many rows as the call has, each pattern at several alignments)
        at = (torch.arange(rows) + first) % len(made)
        op.forward(made[at.cuda()], top_classes=best, top_logprobs=logprobs)
        assert torch.equal(best.cpu().long(), want[at])
    shifted = torch.zeros(rows * (classes + 1) + 3, dtype=made.dtype, device="cuda")[3:].view(rows, classes + 1)[:, :classes]
    at = torch.arange(rows) % len(made)
    shifted.copy_(made[at.cuda()])
    op.forward(shifted, top_classes=best, top_logprobs=logprobs)
    assert torch.equal(best.cpu().long(), want[at])


@pytest.mark.parametrize("kind,rows,classes", CASES)
@pytest.mark.parametrize("top", [1, 5, 64])
def test_logits_of_few_values(kind, rows, classes, top):
    """Clamped logits: many rows share their largest values, and many of a row's logits are equal."""
    import torch
    rows = min(rows, 1100)
    x = (torch.randn(rows, classes, generator=torch.Generator().manual_seed(top)) * 4).round().clamp(-9, 9)
    x[::2, -7:] = 9.0
    x[::3, : classes - 40] = x[::3, : classes - 40].clamp(max=8.0)
    x = x.to(_types()[kind][0]).cuda()
    import paper_2312_08728_amd as B
    op = B.LogProbs(classes, dtype=_types()[kind][1], top=top)
    best, logprobs = torch.empty(rows, top, dtype=torch.int32, device="cuda"), torch.empty(rows, top, device="cuda")
    op.forward(x, top_classes=best, top_logprobs=logprobs)
    want = torch.sort(x.float(), dim=1, descending=True, stable=True)[1][:, :top]
    assert torch.equal(best.long(), want)

@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("classes,top", [(1, 1), (3, 3), (7, 7), (64, 64), (64, 5), (700, 64), (2500, 9), (9001, 3), (40_000, 64), (50_257, 5)])
def test_nan_at_the_first_class(kind, classes, top):
    """NaN comes first, in the order of its classes, class 0 too: rows that are all NaN, that have one at class 0, at class 0 and others, at all classes but 0."""
    import torch
    nan = float("nan")
    x = torch.randn(5, classes, generator=torch.Generator().manual_seed(classes))
    x[0] = nan
    x[1, 0] = nan
    x[2, 0], x[2, classes // 2], x[2, classes - 1] = nan, nan, nan
    x[3, 1:] = nan
    x[4, 0], x[4, classes - 1] = nan, float("inf")
    x = x.to(_types()[kind][0]).cuda()
    _check(kind, x, _labels(5, classes), top)
