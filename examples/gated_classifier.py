"""Buffered mini-batch training of a gated block with AdamW, next to softmax regression on the same buffers.

    python examples/gated_classifier.py [--rows 65536] [--state-bits 8] ...

Algorithm 1 with another predictor and another update: buffers of rows stream from pinned host memory into one of two
slots on the device while the other is computed on; every pass over a buffer draws the partition that the library's own
runs draw (Context.get_perm), and every mini-batch makes a forward pass, the gradient of the mean cross-entropy (LogProbs), a
backward pass and one AdamW step over the weights.  With --norm rows are normed (RMSNorm, with a weight that is trained) before the block.  Masters are fp32; the block multiplies by their bf16 copies,
which the step leaves.  The labels come from a gated block, so that no linear predictor fits them.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2312_08728_amd as B  # noqa: E402


def draw_data(rows, p, classes, seed):
    """Gaussian rows in bf16 and the classes that a random gated block (and Gumbel noise) gives them, on the host, pinned."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    x = normal(rows, p).bfloat16()
    hidden = 2 * p
    gate, up, down = normal(p, hidden) / p ** 0.5, normal(p, hidden) / p ** 0.5, 12.0 * normal(hidden, classes) / hidden ** 0.5
    scores = (torch.sigmoid(4.0 * (x.float() @ gate)) * (x.float() @ up)) @ down
    noise = -torch.log(-torch.log(torch.rand(scores.shape, generator=gen, device="cuda").clamp(1e-7, 1 - 1e-7)))
    y = torch.argmax(scores + noise, 1).int()
    return x.cpu().pin_memory(), y.cpu().pin_memory()


class GatedClassifier:
    """Weights, their gradients and bf16 copies, the block, the log probabilities, the optimizer, and the norm before the block if there is one."""

    def __init__(self, p, hidden, classes, batch, lr, state_bits, seed, norm=False):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        shapes = [(p, hidden), (p, hidden), (hidden, classes)]
        self.masters = [torch.randn(s, generator=gen, device="cuda") / s[0] ** 0.5 for s in shapes] + [torch.ones(p, device="cuda")] * norm
        self.weights = [m.bfloat16() for m in self.masters]
        self.grads = [torch.zeros_like(w) for w in self.weights]
        self.block = B.GatedBlock(p, hidden, classes, batch, dtype=B.BMGD_BF16, activation=B.BMGD_ACT_SILU)
        self.optimizer = B.AdamW(self.masters, self.grads, copies=self.weights, lr=lr, weight_decay=0.01, state_bits=state_bits)
        new = lambda n: torch.empty(batch, n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.y, self.g, self.u = new(classes), new(hidden), new(hidden)
        self.scores = B.LogProbs(classes, dtype=B.BMGD_BF16)
        self.logprob, self.kept = torch.empty(batch, device="cuda"), torch.empty(batch, 3, device="cuda")
        self.norm = B.RMSNorm(p, dtype=B.BMGD_BF16) if norm else None
        if norm:
            self.normed, self.dnormed, self.rstd = new(p), new(p), torch.empty(batch, device="cuda")

    def forward(self, x, stream, keep=False):
        """Logits of the rows x; with `keep` what a backward pass needs stays."""
        n = x.shape[0]
        if self.norm:
            self.norm.forward(x, self.weights[3], y=self.normed[:n], rstd=self.rstd[:n], stream=stream)
            x = self.normed[:n]
        g, u = (self.g[:n], self.u[:n]) if keep else (None, None)
        self.block.forward(x, *self.weights[:3], self.y[:n], g=g, u=u, stream=stream)
        return self.y[:n]

    def step(self, x, labels, lr, stream):
        """One update from the rows x."""
        n = x.shape[0]
        y, kept, rows = self.forward(x, stream, keep=True), self.kept[:n], self.normed[:n] if self.norm else x
        self.scores.forward(y, kept=kept, stream=stream)
        self.scores.backward(y, kept, y, labels=labels, dlogprob=torch.full((n,), -1.0 / n, device="cuda"), stream=stream)     # the logits' gradient takes their place
        dx = self.dnormed[:n] if self.norm else None
        self.block.backward(y, rows, *self.weights[:3], self.g[:n], self.u[:n], dx=dx, dgate=self.grads[0], dup=self.grads[1], ddown=self.grads[2], stream=stream)
        if self.norm:
            self.norm.backward(dx, x, self.weights[3], self.rstd[:n], dx, dweight=self.grads[3], stream=stream)
        self.optimizer.step(lr=lr, stream=stream)

    def loss(self, x, labels, stream):
        """Mean cross-entropy, mini-batch by mini-batch."""
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for xs, ls in zip(x.split(self.y.shape[0]), labels.split(self.y.shape[0])):
            logprob = self.logprob[: xs.shape[0]]
            self.scores.forward(self.forward(xs, stream), labels=ls, logprob=logprob, stream=stream)
            total -= logprob.double().sum()
        return float(total) / x.shape[0]


def train(rows=65_536, p=128, hidden=512, classes=10, buffers=4, batch=1_024, passes=2, iterations=4, lr=3e-3, state_bits=32, seed=0, norm=False, say=print):
    """Returns (losses of the gated block after every iteration over the buffers, loss of softmax regression after the last one)."""
    host_x, host_y = draw_data(rows, p, classes, seed)
    per = -(-rows // buffers)
    buffers = -(-rows // per)                               # as many as have rows
    slots = [(torch.empty(per, p, dtype=torch.bfloat16, device="cuda"), torch.empty(per, dtype=torch.int32, device="cuda")) for _ in range(2)]
    copy, compute = torch.cuda.Stream(), torch.cuda.Stream()
    loaded = [torch.cuda.Event() for _ in slots]
    read = [torch.cuda.Event() for _ in slots]
    model = GatedClassifier(p, hidden, classes, batch, lr, state_bits, seed + 1, norm)
    # softmax regression on the same buffers; also the source of the partitions
    linear = B.Context(p, per, batch, 0.5, passes, model=B.BMGD_SOFTMAX, n_classes=classes, seed=seed)
    torch.cuda.synchronize()

    updates = iterations * passes * sum(-(-min(per, rows - k * per) // batch) for k in range(buffers))
    done, losses = 0, []

    def load(k):
        slot, first = k % 2, (k % buffers) * per
        n = min(per, rows - first)
        copy.wait_event(read[slot])
        with torch.cuda.stream(copy):
            slots[slot][0][:n].copy_(host_x[first:first + n], non_blocking=True)
            slots[slot][1][:n].copy_(host_y[first:first + n], non_blocking=True)
            loaded[slot].record()
        return n

    with torch.cuda.stream(compute):
        n = load(0)
        for k in range(iterations * buffers):
            slot, rows_here = k % 2, n
            if k + 1 < iterations * buffers:
                n = load(k + 1)                             # the buffering step of the next buffer
            compute.wait_event(loaded[slot])
            x, y = slots[slot][0][:rows_here], slots[slot][1][:rows_here]
            for t in range(1, passes + 1):
                order = torch.from_numpy(linear.get_perm(k, t, rows_here)).cuda()
                for pick in order.split(batch):
                    # the rate falls to a tenth of its value
                    model.step(x.index_select(0, pick), y.index_select(0, pick), lr * (1.0 - 0.9 * done / updates), compute)
                    done += 1
            linear.run_device_buffer(x, y, rows_here, compute)
            read[slot].record()
            if (k + 1) % buffers == 0:
                losses.append(model.loss(host_x.cuda(), host_y.cuda(), compute))
                say(f"iteration {(k + 1) // buffers}: mean cross-entropy {losses[-1]:.4f}")
        compute.synchronize()
        reference = linear.eval_loss(host_x.cuda(), host_y.cuda(), rows, compute)
        say(f"softmax regression on the same buffers: {reference:.4f}")
    model.block.close()
    linear.close()
    return losses, reference


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("rows", 65_536), ("p", 128), ("hidden", 512), ("classes", 10), ("buffers", 4), ("batch", 1_024), ("passes", 2), ("iterations", 4),
                        ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--lr", type=float, default=3e-3)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    ap.add_argument("--norm", action="store_true", help="norm rows before the block")
    train(**{k: v for k, v in vars(ap.parse_args()).items()})


if __name__ == "__main__":
    main()
