"""Norm, gated block, 8-bit product, log probabilities and AdamW as a program runs them: one after the other, on streams, captured."""
import math
import threading

import numpy as np
import pytest

from oracle import operators as O
from test_gpu_gated_example import _example
from test_gpu_logprobs import E, _close, _np, _sum_error
from test_gpu_network_streams import _busy, _marker

pytestmark = pytest.mark.gpu


def _bf16(*shape, seed=0, scale=1.0):
    import torch
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16().cuda()


class _Served:
    """A row's way: residual and norm into 8 bits, a layer in 8 bits, the most probable classes."""

    def __init__(self, rows, p, classes, top):
        import torch
        import paper_2312_08728_amd as B
        self.norm, self.layer, self.scores = B.RMSNorm(p), B.Int8Product(p, classes), B.LogProbs(classes, top=top)
        self.weight, layer = _bf16(p, seed=3, scale=0.2) + 1, _bf16(p, classes, seed=4, scale=p ** -0.5)
        byte, f, i = (lambda *s: torch.empty(*s, dtype=torch.int8, device="cuda")), (lambda *s: torch.empty(*s, device="cuda")), lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")
        self.w, self.w_scales = byte(classes, p), f(classes)
        self.layer.quantize(layer, self.w, self.w_scales)
        self.codes, self.scales, self.y = byte(rows, p), f(rows), torch.empty(rows, classes, dtype=torch.bfloat16, device="cuda")
        self.logprob, self.entropy, self.top_classes, self.top_logprobs = f(rows), f(rows), i(rows, top), f(rows, top)
        torch.cuda.synchronize()

    def __call__(self, x, residual, labels, stream=None):
        self.norm.forward(x, self.weight, residual=residual, sum=residual, codes=self.codes, scales=self.scales, stream=stream)
        self.layer.forward(self.codes, self.scales, self.w, self.w_scales, self.y, stream=stream)
        self.scores.forward(self.y, labels=labels, logprob=self.logprob, entropy=self.entropy, top_classes=self.top_classes, top_logprobs=self.top_logprobs, stream=stream)
        return self.y, self.logprob, self.entropy, self.top_classes, self.top_logprobs


@pytest.mark.parametrize("rows,p,classes,top", [(1, 512, 1000, 5), (3, 123, 40_001, 20), (77, 640, 1000, 3), (300, 1365, 130, 64)])
def test_served_in_8_bits(rows, p, classes, top):
    import torch
    x, r = _bf16(rows, p, seed=1), _bf16(rows, p, seed=2)
    labels = torch.arange(rows, dtype=torch.int32, device="cuda") % classes
    served = _Served(rows, p, classes, top)
    s = (x.float() + r.float()).bfloat16()
    y, logprob, entropy, top_classes, top_logprobs = served(x, r, labels)
    assert torch.equal(r, s)
    codes, largest = O.codes_of(_np(s) * _np(served.weight))
    assert (served.codes.cpu().numpy() == codes).all()
    total = torch.from_numpy(codes).double() @ served.w.cpu().double().t()
    assert torch.equal(y.cpu(), (total.float() * served.scales.cpu()[:, None] * served.w_scales.cpu()).bfloat16())
    # the logits are off from those of the layer's own weights by the codes' roundings: half a step each
    own = _np(s) * _np(served.weight) / np.sqrt((_np(s) ** 2).mean(1, keepdims=True) + 1e-6)
    layer = _np(_bf16(p, classes, seed=4, scale=p ** -0.5))
    step_x, step_w = np.abs(own).max(1, keepdims=True) / 127, np.abs(layer).max(0, keepdims=True) / 127
    bound = 0.5 * step_x * np.abs(layer).sum(0) + 0.5 * step_w * np.abs(own).sum(1, keepdims=True) + 0.25 * p * step_x * step_w
    want = own @ layer
    assert (np.abs(_np(y) - want) <= bound * 1.001 + np.abs(want) * 2.0 ** -8 + 1e-5).all()
    logits = _np(y)
    logp, h = O.log_probabilities(logits)
    k = _sum_error(classes)
    lp = logp[np.arange(rows), np.arange(rows) % classes]
    _close(logprob, lp, E * (2 * np.abs(lp) + k))
    _close(entropy, h, E * (k + 16) * (1 + math.log(classes + 1)))
    best = O.best(logits, top)
    assert (top_classes.cpu().numpy() == best).all()
    want = np.take_along_axis(logp, best, 1)
    _close(top_logprobs, want, E * (2 * np.abs(want) + k))


def test_a_captured_answer():
    """The whole way in one graph, replayed on other rows, with eager calls and synchronizations between the replays."""
    import torch
    rows, p, classes = 2, 256, 70_000                           # (several workgroups for a row, with a workspace)
    served, eager = _Served(rows, p, classes, 9), _Served(rows, p, classes, 9)
    x, r, labels = _bf16(rows, p, seed=1), _bf16(rows, p, seed=2), torch.zeros(rows, dtype=torch.int32, device="cuda")
    served(x, r, labels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = served(x, r, labels)
    for seed in range(4):
        x.copy_(_bf16(rows, p, seed=10 + seed))
        r.copy_(_bf16(rows, p, seed=20 + seed))
        r2 = r.clone()
        labels.fill_(seed)
        graph.replay()
        want = eager(x, r2, labels)
        torch.cuda.synchronize()
        assert torch.equal(r, r2) and all(torch.equal(a, b) for a, b in zip(out, want))


def test_a_training_step_eager_and_captured():
    """Norm, block, log probabilities and back, then AdamW: a captured step makes what the same eager calls make, bit by bit."""
    import torch
    import paper_2312_08728_amd as B
    rows, p, hidden, classes = 1500, 96, 160, 50

    def made():
        m = _example().GatedClassifier(p, hidden, classes, rows, 1e-2, 32, 5, norm=True)
        return m, _bf16(rows, p, seed=1), torch.arange(rows, dtype=torch.int32, device="cuda") % classes
    (a, xa, la), (b, xb, lb) = made(), made()
    f = torch.full((rows,), -1.0 / rows, device="cuda")

    def gradients(m, x, labels):
        """The step without its update (an update holds its number)."""
        y = m.forward(x, None, keep=True)
        m.scores.forward(y, labels=labels, logprob=m.logprob, kept=m.kept)
        m.scores.backward(y, m.kept, y, labels=labels, dlogprob=f)
        m.block.backward(y, m.normed, *m.weights[:3], m.g, m.u, dx=m.dnormed, dgate=m.grads[0], dup=m.grads[1], ddown=m.grads[2])
        m.norm.backward(m.dnormed, x, m.weights[3], m.rstd, m.dnormed, dweight=m.grads[3])
    gradients(a, xa, la)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gradients(a, xa, la)
    for seed in range(3):
        for x in (xa, xb):
            x.copy_(_bf16(rows, p, seed=30 + seed))
        graph.replay()
        a.optimizer.step()
        gradients(b, xb, lb)
        b.optimizer.step()
        torch.cuda.synchronize()
        for s, t in zip((*a.masters, *a.grads, a.logprob, a.dnormed), (*b.masters, *b.grads, b.logprob, b.dnormed)):
            assert torch.equal(s, t)
    for m in (a, b):
        m.block.close()


def test_gradients_of_the_whole_way():
    """Of the mean cross-entropy, against torch's own in 64 bits.  Every stage rounds to 16 bits (half a step 2^-8, relative): the norm's rows, G, U and H, the logits,
    their gradient, dG and dU, the block's dX and the results; what is added up has both signs, so the error is compared in the Euclidean norm, where each
    stage adds at most twice its half step (a factor between the derivative's and the value's) and ten stages stay below 20 x 2^-8."""
    import torch
    rows, p, hidden, classes = 200, 64, 128, 30
    m = _example().GatedClassifier(p, hidden, classes, rows, 1e-2, 32, 5, norm=True)
    x, labels = _bf16(rows, p, seed=1), torch.arange(rows, dtype=torch.int32, device="cuda") % classes
    m.optimizer.step = lambda **kw: None                        # gradients only
    m.step(x, labels, 0.0, None)
    w = [t.double().cpu().requires_grad_() for t in m.weights]
    s = x.double().cpu()
    n = s * torch.rsqrt((s * s).mean(1, keepdim=True) + 1e-6) * w[3]
    y = (torch.nn.functional.silu(n @ w[0]) * (n @ w[1])) @ w[2]
    torch.nn.functional.cross_entropy(y, labels.long().cpu()).backward()
    for g, t in zip(m.grads, w):
        assert float((g.double().cpu() - t.grad).norm() / t.grad.norm()) <= 20 * 2.0 ** -8
    m.block.close()


def test_the_example_with_a_norm():
    losses, linear = _example().train(rows=5_003, p=40, hidden=72, classes=7, buffers=2, batch=333, passes=1, iterations=2, norm=True, say=lambda s: None)
    assert len(losses) == 2 and all(math.isfinite(v) for v in (*losses, linear))


def test_calls_follow_the_stream_they_are_made_on():
    """Behind a busy stream, as the current one and by name; what a call needs besides lies where nothing else writes meanwhile."""
    import torch
    import paper_2312_08728_amd as B
    rows, classes, n = 2, 200_000, 1000
    x = torch.randn(rows, classes, device="cuda")
    late = torch.zeros_like(x)
    op, norm = B.LogProbs(classes, dtype=B.BMGD_F32, top=7), B.RMSNorm(n, dtype=B.BMGD_F32)
    dy, s, w = torch.randn(4000, n, device="cuda"), torch.randn(4000, n, device="cuda"), torch.randn(n, device="cuda")
    assert B.bmgd_logprobs_workspace_bytes(op.cfg, rows) and B.bmgd_norm_workspace_bytes(norm.cfg, 4000)

    def new():
        f = lambda *k: torch.zeros(*k, device="cuda")  # noqa: E731
        return dict(entropy=f(rows), kept=f(rows, 3), top_classes=f(rows, 7).int(), top_logprobs=f(rows, 7)), f(4000, n), f(n)
    rstd = torch.rand(4000, device="cuda")
    want, dx, dw = new()
    op.forward(x, **want)
    norm.backward(dy, s, w, rstd, dx, dweight=dw)
    torch.cuda.synchronize()
    for way in ("current", "named"):
        stream = torch.cuda.Stream()
        out, dx2, dw2 = new()
        late.zero_()
        torch.cuda.synchronize()
        _busy(stream)
        with torch.cuda.stream(stream):
            late.copy_(x)
            if way == "current":
                op.forward(late, **out)
                norm.backward(dy, s, w, rstd, dx2, dweight=dw2)
        if way == "named":
            op.forward(late, **out, stream=stream)
            norm.backward(dy, s, w, rstd, dx2, dweight=dw2, stream=stream.cuda_stream)
        end = _marker(stream)
        others = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(32)]          # (memory that torch has free on this stream)
        assert not end.query()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in want) and torch.equal(dx2, dx) and torch.equal(dw2, dw)
        del others


def test_two_threads_at_once():
    """One object for both, a stream each."""
    import torch
    import paper_2312_08728_amd as B
    rows, classes = 3, 50_000
    op = B.LogProbs(classes, top=5)
    xs = [_bf16(rows, classes, seed=i) for i in range(2)]
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")

    def run(x, into):
        out = dict(logprob=torch.empty(rows, device="cuda"), top_classes=torch.empty(rows, 5, dtype=torch.int32, device="cuda"), top_logprobs=torch.empty(rows, 5, device="cuda"))
        op.forward(x, labels=labels, **out)
        into.append(out)
    want, got = [], [[], []]
    for x in xs:
        run(x, want)
    torch.cuda.synchronize()

    def many(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(50):
                run(xs[i], got[i])
        s.synchronize()
    threads = [threading.Thread(target=many, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        assert len(got[i]) == 50 and all(torch.equal(o[k], want[i][k]) for o in got[i] for k in o)


def test_results_are_told_to_autograd():
    import torch
    import paper_2312_08728_amd as B
    x = torch.zeros(4, 16, dtype=torch.bfloat16, device="cuda").detach()
    before = x._version
    y, c, s = torch.zeros_like(x), torch.zeros(4, 16, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    B.RMSNorm(16).forward(x, y=y, codes=c, scales=s)
    assert x._version == before and (y._version, c._version, s._version) == (1, 1, 1)
