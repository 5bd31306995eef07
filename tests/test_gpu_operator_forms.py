"""Every form of the kernels that the rules choose, against 64-bit forms: one shape at least for each, and a test of which form a shape gets, so that a rule that changes cannot leave
one without a test.  (Shapes for 256 compute units; pieces of 16 bytes decide, so fp32 rows have half the columns of 16-bit ones.)
"""
import json
import os
import re
import subprocess
import sys

import numpy as np
import pytest

import test_gpu_int8 as I
import test_gpu_logprobs as L
import test_gpu_norm as N

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (rows, p, out) -> form.  p a multiple of 16: rows at whole pieces, any other: loose
PRODUCT = {
    (4096, 208, 4096): "tile 256 256 2 4 1 false", (2049, 272, 2111): "tile 128 128 2 2 1 false", (1000, 272, 2050): "tile 128 128 2 2 2 false", (1590, 528, 1010): "tile 64 128 2 2 2 false",
    (700, 304, 1001): "tile 64 64 2 4 3 false", (300, 256, 300): "tile 32 32 2 2 4 false", (5, 1040, 50): "few 1", (17, 2048, 4097): "few 2", (33, 4096, 4097): "few 4",
    (2100, 77, 2300): "tile 128 128 2 2 1 true", (1000, 273, 2056): "tile 128 128 2 4 2 true", (513, 333, 1001): "tile 64 64 2 4 4 true", (333, 1365, 1000): "tile 32 64 2 2 4 true",
    (300, 513, 100): "tile 32 32 2 2 6 true", (200, 777, 150): "few 1", (4, 1041, 16): "few 1", (17, 513, 1000): "few 2", (33, 1041, 1000): "few 4",
}
# (rows, fp32 classes, top, entropy) -> form
SCORES = {
    (1030, 1301, 0, True): "1 false true", (1030, 5001, 0, True): "1 false true", (1030, 8001, 0, False): "1 false false", (1030, 2001, 5, True): "1 true true", (1030, 2001, 16, False): "1 true false",
    (1030, 350, 64, True): "1 true true", (1030, 350, 64, False): "1 true false", (40, 10_003, 0, True): "4 false true join", (300, 10_003, 0, True): "4 false true",
    (300, 10_003, 0, False): "4 false false", (1030, 5001, 5, True): "4 true true", (300, 10_003, 20, False): "4 true false", (40, 10_003, 20, False): "4 true false join", (3, 30_001, 9, True): "4 true true join", (3, 30_001, 9, False): "4 true false join", (3, 30_001, 0, False): "4 false false join",
}
# (rows, fp32 columns) -> form with dw, form without.  Rows for several turns of a workgroup
NORM = {
    (9000, 300): ("1 2 1", "1 2 0"), (9000, 100): ("1 1 1", "1 1 0"), (3000, 1024): ("4 1 1", "4 1 0"), (2100, 683): ("4 1 1", "4 1 0"), (2100, 2048): ("4 2 1", "4 2 0"), (1100, 4000): ("4 4 1", "4 4 0"),
    (700, 8192): ("16 2 1", "16 2 0"), (1000, 300): ("1 2 2", "1 2 0"), (1000, 1024): ("4 1 2", "4 1 0"), (500, 2048): ("4 2 2", "4 2 0"),
}

CHILD = """
import json, torch
import paper_2312_08728_amd as B
from torch.profiler import profile, ProfilerActivity
from test_gpu_operator_forms import NORM, PRODUCT, SCORES
F = B.BMGD_F32
f = lambda *s: torch.zeros(*s, device="cuda")
byte = lambda *s: torch.zeros(*s, dtype=torch.int8, device="cuda")
def names(call):
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    return [e.name for e in p.events() if "_kernel" in e.name]
out = [torch.cuda.get_device_properties(0).multi_processor_count, [], [], []]
for rows, p, n in PRODUCT:
    x, w, y, sx, sw = byte(rows, p), byte(n, p), f(rows, n), f(rows), f(n)
    out[1].append(names(lambda: B.Int8Product(p, n, dtype=F).forward(x, sx, w, sw, y)))
for rows, classes, top, entropy in SCORES:
    x, lp, h, b, bl = f(rows, classes), f(rows), f(rows), f(rows, top).int(), f(rows, top)
    labels = lp.int()
    out[2].append(names(lambda: B.LogProbs(classes, dtype=F, top=top).forward(x, labels=labels, logprob=lp, entropy=h if entropy else None, top_classes=b if top else None, top_logprobs=bl if top else None)))
for rows, n in NORM:
    s, dx, r, w, dw = f(rows, n), f(rows, n), f(rows), f(n), f(n)
    op, dy = B.RMSNorm(n, dtype=F), f(rows, n)
    out[3].append([names(lambda: op.backward(dy, s, w, r, dx, dweight=dw)), names(lambda: op.backward(dy, s, w, r, dx))])
print("FORMS", json.dumps(out))
"""


def _form(name):
    """`int8_tile_kernel<float, (anonymous namespace)::Tile<128, ...> >(...)` -> (int8_tile, "128 ...")."""
    kernel, arguments = re.search(r"(\w+)_kernel<float(.*)>\(", name).groups()
    return kernel, " ".join(re.findall(r"\b(?:\d+|true|false)\b", arguments))


def test_forms_that_shapes_get():
    """In a process of its own, under torch's profiler."""
    path = os.pathsep.join([ROOT, os.path.join(ROOT, "tests"), os.environ.get("PYTHONPATH", "")])
    done = subprocess.run([sys.executable, "-c", CHILD], env={**os.environ, "PYTHONPATH": path}, cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-2000:]
    units, product, scores, norm = json.loads(done.stdout.split("FORMS ", 1)[1])
    if units != 256:
        pytest.skip("the rules go by compute units, and these shapes by 256 of them")
    if not any(product):
        pytest.skip("torch's profiler names no kernels here")
    for shape, found in zip(PRODUCT, product):
        (kernel, arguments), = [_form(n) for n in found]
        assert f"{kernel[5:]} {arguments}" == PRODUCT[shape], shape
    for shape, found in zip(SCORES, scores):
        forms = [_form(n) for n in found]
        assert forms[0][0] == "logprobs" and forms[0][1] + " join" * (len(forms) == 2) == SCORES[shape], shape
    for shape, found in zip(NORM, norm):
        assert tuple(next(a for k, a in map(_form, f) if k == "norm_backward") for f in found) == NORM[shape], shape


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,p,out", PRODUCT)
def test_product(kind, rows, p, out):
    I._check(rows, p, out, kind, pads=(0, 0, 3))


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,classes,top,entropy", SCORES)
def test_scores(kind, rows, classes, top, entropy):
    """With entropy all results, compared at some rows of all; without, the same bits as with it, and both the definition's."""
    import torch
    import paper_2312_08728_amd as B
    classes = classes if kind == "f32" else 2 * classes - 1
    x, _ = L._logits(rows, classes, L._types()[kind][0], pad=1, seed=top)
    labels = L._labels(rows, classes)
    gpu = torch.from_numpy(labels).int().cuda()
    op, out = L._forward(kind, x, gpu, top)
    if not entropy:
        part = {k: torch.full_like(v, 7) for k, v in out.items() if k in ("logprob", "top_classes", "top_logprobs")}
        op.forward(x, labels=gpu, **part)
        assert all(torch.equal(part[k], out[k]) for k in part)
    at = slice(0, rows, -(-rows // 64))
    x64, labels = L._np(x[at]), labels[at]
    logp, h = L.O.log_probabilities(x64)
    k = L._sum_error(classes)
    chosen = np.where(labels < 0, 0.0, logp[np.arange(len(labels)), np.clip(labels, 0, None)])
    L._close(out["logprob"][at], chosen, L.E * (2 * np.abs(chosen) + k))
    L._close(out["entropy"][at], h, L.E * (k + 16) * (1 + np.log(classes + 1)))
    if top:
        best = L.O.best(x64, top)
        assert (out["top_classes"][at].cpu().numpy() == best).all()
        want = np.take_along_axis(logp, best, 1)
        L._close(out["top_logprobs"][at], want, L.E * (2 * np.abs(want) + k))
        # (and every row's classes, by a stable sort)
        assert torch.equal(out["top_classes"].long(), torch.sort(x.float(), dim=1, descending=True, stable=True)[1][:, :top])


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,n", NORM)
@pytest.mark.parametrize("way", ["all", "plain"])
def test_norm_backward(kind, rows, n, way):
    N.test_backward(kind, rows, n if kind == "f32" or n % 2 else 2 * n, 0, way)
