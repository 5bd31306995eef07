"""Speed and results of the operators around a gated block: root-mean-square norm, 8-bit product, log probabilities.

The norm adds a residual, norms the sum and writes it in 16 bits, or as 8-bit codes with a scale for each row; backward
from dY.  The product multiplies such codes by a layer's codes, which have a scale for each of its outputs.  Log
probabilities are those of given classes, with the entropy and the most probable classes, as a server answers; and with
their gradient, as a training step needs it.

`own` false: elementary torch operations in 32 bits (8-bit codes, which lie next to borders, in 64), rounded once at the
end.  `own` true: the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
TINY = 2.0 ** -118          # a row whose largest weighted value is below this is held as zeros


def _norm(name, rows, n, dtype="bf16", residual=True, bits=16):
    case = {"kind": "norm", "rows": rows, "n": n, "dtype": dtype, "residual": residual, "bits": bits}
    return case if name is None else {"name": name, **case}


def _norm_backward(name, rows, n, dtype="bf16", residual=True):
    case = {"kind": "norm_backward", "rows": rows, "n": n, "dtype": dtype, "residual": residual}
    return case if name is None else {"name": name, **case}


def _product(name, rows, p, out, dtype="bf16"):
    case = {"kind": "product", "rows": rows, "p": p, "out": out, "dtype": dtype}
    return case if name is None else {"name": name, **case}


def _scores(name, kind, rows, classes, dtype="bf16", top=0, padded=False):
    case = {"kind": kind, "rows": rows, "classes": classes, "dtype": dtype, "top": top, "padded": padded}
    return case if name is None else {"name": name, **case}


def listed():
    return [
        # one row on its way to an 8-bit product: latency is all there is
        _norm("norm_8bit_one_row", rows=1, n=4_096, bits=8),
        # training forward with nothing a multiple of anything
        _norm("norm_ragged", rows=777, n=1_365, dtype="f16"),
        # 8-bit operands of a large product
        _norm("norm_8bit_large", rows=8_192, n=8_192, bits=8),
        # backward of a mini-batch of 1,000 rows of 512 detector features, in 32 bits
        _norm_backward("norm_backward_small", rows=1_000, n=512, dtype="f32", residual=False),
        # backward of a mini-batch of 8,192 rows of 4,096 features, with the gradient that comes along the residual
        _norm_backward("norm_backward_large", rows=8_192, n=4_096),
        # one row is answered: 34 MB of weights stream past it
        _product("product_one_row", rows=1, p=4_096, out=8_192),
        # a batch of rows that arrived together, odd widths
        _product("product_ragged", rows=333, p=1_365, out=1_000, dtype="f16"),
        # a mini-batch of 8,192 rows
        _product("product_large", rows=8_192, p=4_096, out=8_192),
        # one row of 1,000 classes is answered with its five most probable ones
        _scores("logprobs_one_row", "score", rows=1, classes=1_000, top=5),
        # a few rows of many classes, in 32 bits, twenty alternatives; the last classes are padding
        _scores("logprobs_few_rows", "score", rows=16, classes=100_003, dtype="f32", top=20, padded=True),
        # a large batch is scored: 0.5 GB of logits
        _scores("logprobs_large", "score", rows=8_192, classes=32_000, top=8),
        # training step: log probabilities and the gradient of their mean with an entropy term, some rows left out
        _scores("logprobs_gradient", "train", rows=4_097, classes=10_001, dtype="f16", padded=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_backward", "product", "product", "score", "score", "train"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    suited = rng.random() < 0.5                 # widths that suit the machine, as most models have
    width = lambda lo, hi: -(-_log_int(rng, lo, hi) // 64) * 64 if suited else _log_int(rng, lo, hi)  # noqa: E731
    rows = _log_int(rng, 1, 8_192)
    if kind == "norm":
        return _norm(None, rows, width(64, 8_192), dtype, rng.random() < 0.7, rng.choice([16, 8]))
    if kind == "norm_backward":
        return _norm_backward(None, rows, width(64, 8_192 if dtype != "f32" else 4_096), dtype, rng.random() < 0.7)
    if kind == "product":
        return _product(None, rows, width(64, 8_192), width(64, 4_096), dtype)
    most = 8_192 * 32_000 // (2 if dtype == "f32" else 1) // (4 if kind == "train" else 1)
    classes = width(10, 131_072)
    rows = min(rows, max(1, most // classes))
    return _scores(None, kind, rows, classes, dtype, 0 if kind == "train" else min(classes // 2, rng.choice([0, 1, 5, 20, 64])), rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _handle(case):
    """What a program keeps between calls."""
    if not own:
        return None
    import paper_2312_08728_amd as B
    dtype = {"bf16": B.BMGD_BF16, "f16": B.BMGD_F16, "f32": B.BMGD_F32}[case["dtype"]]
    if case["kind"] in ("norm", "norm_backward"):
        return B.RMSNorm(case["n"], dtype=dtype, eps=EPS)
    if case["kind"] == "product":
        return B.Int8Product(case["p"], case["out"], dtype=dtype)
    return B.LogProbs(case["classes"], dtype=dtype, top=case["top"])


def _row_codes(v):
    """8-bit codes and scales of the rows of a float matrix: v = scale * code, scale = the row's largest / 127."""
    scale = v.abs().amax(1) / 127.0
    return torch.round(v / scale[:, None]).clamp(-127.0, 127.0).to(torch.int8), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, rows, dtype = case["kind"], case["rows"], TYPES[case["dtype"]]
    new = lambda *shape, dtype=dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731

    def normal(*shape, scale=1.0, shift=0.0, dtype=dtype):
        return (torch.randn(shape, generator=gen, device="cuda") * scale + shift).to(dtype)

    state = {"case": case, "handle": _handle(case)}
    if kind in ("norm", "norm_backward"):
        n = case["n"]
        # rows of different sizes, a few features much larger than the others, as a residual stream has them
        size = torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device="cuda")) * (1.0 + 9.0 * (torch.rand(1, n, generator=gen, device="cuda") < 0.01))
        state["x"] = (torch.randn(rows, n, generator=gen, device="cuda") * size).to(dtype)
        state["weight"] = normal(n, scale=0.2, shift=1.0)
        if kind == "norm":
            state["residual"] = (torch.randn(rows, n, generator=gen, device="cuda") * size).to(dtype) if case["residual"] else None
            state["sum"] = new(rows, n) if case["residual"] else None
            if case["bits"] == 8:
                state["codes"], state["scales"], state["values"] = new(rows, n, dtype=torch.int8), new(rows, dtype=torch.float32), new(rows, n, dtype=torch.float32)
            else:
                state["y"] = new(rows, n)
        else:
            # x: the sum that the forward pass has kept
            state["rstd"] = 1.0 / torch.sqrt(state["x"].float().square().mean(1) + EPS)
            state["dy"] = normal(rows, n)
            state["dsum"] = normal(rows, n) if case["residual"] else None
            state["dx"], state["dweight"] = new(rows, n), new(n)
    elif kind == "product":
        p, out = case["p"], case["out"]
        state["x"], state["x_scales"] = _row_codes(normal(rows, p, dtype=torch.float32))
        state["w"], state["w_scales"] = _row_codes(normal(out, p, scale=p ** -0.5, dtype=torch.float32))
        state["y"] = new(rows, out)
    else:
        classes, top = case["classes"], case["top"]
        real = classes - classes // 16 if case["padded"] else classes       # those behind are padding
        state["logits"] = normal(rows, classes, scale=2.5)
        state["logits"][:, real:] = -math.inf
        state["labels"] = torch.randint(0, real, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        state["logprob"], state["entropy"] = new(rows, dtype=torch.float32), new(rows, dtype=torch.float32)
        if kind == "score":
            state["top_classes"] = new(rows, top, dtype=torch.int32) if top else None
            state["top_logprobs"] = new(rows, top, dtype=torch.float32) if top else None
        else:
            left_out = torch.rand(rows, generator=gen, device="cuda") < 0.1
            state["labels"] = torch.where(left_out, torch.full_like(state["labels"], -1), state["labels"])
            # a loss scale times the mean over the rows, an entropy term of a hundredth of it
            state["dlogprob"] = torch.full((rows,), -1.0, device="cuda")
            state["dentropy"] = torch.full((rows,), -0.01, device="cuda")
            state["kept"] = new(rows, 3, dtype=torch.float32)
            state["dlogits"] = new(rows, classes)
    return state


# ---- the plain forms --------------------------------------------------------------------------------------------------
def _plain_norm(state):
    case = state["case"]
    dtype, out = TYPES[case["dtype"]], {}
    s = state["x"].float()
    if case["residual"]:
        out["sum"] = (s + state["residual"].float()).to(dtype)       # what the stream goes on with is what is normed
        s = out["sum"].float()
    rstd = 1.0 / torch.sqrt((s * s).mean(1) + EPS)
    if case["bits"] == 16:
        out["y"] = (s * state["weight"].float() * rstd[:, None]).to(dtype)
        return out
    v = s.double() * state["weight"].double()
    top = v.abs().amax(1)
    held = top >= TINY
    code = torch.where(held[:, None], torch.round(v * torch.where(held, 127.0 / top, torch.zeros_like(top))[:, None]), torch.zeros_like(v))
    scale = torch.where(held, top.float() * rstd / 127.0, torch.zeros_like(rstd))
    out["values"] = code.float() * scale[:, None]
    return out


def _plain_norm_backward(state):
    dtype = TYPES[state["case"]["dtype"]]
    s, w, dy, rstd = state["x"].float(), state["weight"].float(), state["dy"].float(), state["rstd"][:, None]
    hat = s * rstd
    d = dy * w
    dx = rstd * (d - hat * (d * hat).mean(1, keepdim=True))
    if state["dsum"] is not None:
        dx = dx + state["dsum"].float()
    return {"dx": dx.to(dtype), "dweight": (dy * hat).sum(0).to(dtype)}


def _plain_product(state):
    # (sums of 8-bit products stay far below 2^24 here, so that 32 bits hold them)
    y = state["x"].float() @ state["w"].float().t()
    return {"y": (y * state["x_scales"][:, None] * state["w_scales"]).to(state["y"].dtype)}


def _plain_scores(state):
    case = state["case"]
    x = state["logits"].float()
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    logp = x - m - torch.log(total)
    p = e / total
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    label = state["labels"].long()
    chosen = torch.where(label >= 0, logp.gather(1, label.clamp(min=0)[:, None])[:, 0], torch.zeros_like(entropy))
    out = {"logprob": chosen, "entropy": entropy}
    if case["kind"] == "score":
        if case["top"]:
            order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :case["top"]]
            out["top_classes"], out["top_logprobs"] = order.int(), logp.gather(1, order)
        return out
    dl = torch.where(label >= 0, state["dlogprob"], torch.zeros_like(chosen))
    d = -p * dl[:, None] - state["dentropy"][:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), torch.zeros_like(p))
    d.scatter_add_(1, label.clamp(min=0)[:, None], dl[:, None])
    out["dlogits"] = d.to(state["dlogits"].dtype)
    return out


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(state):
    case, kind, op = state["case"], state["case"]["kind"], state["handle"]
    if not own:
        return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "product": _plain_product}.get(kind, _plain_scores)(state)
    if kind == "norm":
        out = {} if state["sum"] is None else {"sum": state["sum"]}
        if case["bits"] == 16:
            op.forward(state["x"], state["weight"], y=state["y"], residual=state["residual"], sum=state["sum"])
            return {**out, "y": state["y"]}
        op.forward(state["x"], state["weight"], codes=state["codes"], scales=state["scales"], residual=state["residual"], sum=state["sum"])
        op.values(state["codes"], state["scales"], state["values"])          # what the 8 bits stand for
        return {**out, "values": state["values"]}
    if kind == "norm_backward":
        op.backward(state["dy"], state["x"], state["weight"], state["rstd"], state["dx"], dweight=state["dweight"], dsum=state["dsum"])
        return {"dx": state["dx"], "dweight": state["dweight"]}
    if kind == "product":
        op.forward(state["x"], state["x_scales"], state["w"], state["w_scales"], state["y"])
        return {"y": state["y"]}
    out = {"logprob": state["logprob"], "entropy": state["entropy"]}
    if kind == "score":
        op.forward(state["logits"], labels=state["labels"], logprob=state["logprob"], entropy=state["entropy"],
                   top_classes=state["top_classes"], top_logprobs=state["top_logprobs"])
        return {**out, "top_classes": state["top_classes"], "top_logprobs": state["top_logprobs"]} if case["top"] else out
    op.forward(state["logits"], labels=state["labels"], logprob=state["logprob"], entropy=state["entropy"], kept=state["kept"])
    op.backward(state["logits"], state["kept"], state["dlogits"], labels=state["labels"], dlogprob=state["dlogprob"], dentropy=state["dentropy"])
    return {**out, "dlogits": state["dlogits"]}


def work(case):
    """Each input read once and each output written once.  Norms into 8 bits: the norm (codes out) and then the values that the
    codes stand for (codes in, 32 bits out).  A training step reads its logits once: the gradient needs nothing else."""
    item, rows, kind = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]], case["rows"], case["kind"]
    if kind == "norm":
        each = item * (3 if case["residual"] else 1) + (item if case["bits"] == 16 else 1 + 1 + 4)
        return {"bytes": rows * case["n"] * each + item * case["n"] + (8 * rows if case["bits"] == 8 else 0), "flops": 6 * rows * case["n"]}
    if kind == "norm_backward":
        return {"bytes": rows * case["n"] * item * (4 if case["residual"] else 3) + 2 * item * case["n"] + 4 * rows, "flops": 10 * rows * case["n"]}
    if kind == "product":
        p, out = case["p"], case["out"]
        return {"bytes": rows * p + out * p + item * rows * out + 4 * (rows + out), "flops": 2 * rows * p * out}
    elements = rows * case["classes"]
    if kind == "score":
        return {"bytes": item * elements + 12 * rows + 8 * rows * case["top"], "flops": 6 * elements}
    return {"bytes": 2 * item * elements + 20 * rows, "flops": 12 * elements}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        out, s = {}, state["x"].double()
        if case["residual"]:
            out["sum"] = s + state["residual"].double()
            s = out["sum"].to(TYPES[case["dtype"]]).double()        # (exact in 64 bits, so this is the one rounding of the definition)
        root = (s.pow(2).sum(1, keepdim=True) / case["n"] + EPS).sqrt()
        v = torch.mul(s, state["weight"].double())
        if case["bits"] == 16:
            return {**out, "y": v / root}
        top = v.abs().max(1, keepdim=True).values
        code = torch.where(top < TINY, torch.zeros_like(v), (v * (127.0 / top.clamp(min=TINY))).round())
        return {**out, "values": code * top / (127.0 * root)}
    if kind == "norm_backward":
        s, w, dy, r = state["x"].double(), state["weight"].double(), state["dy"].double(), state["rstd"].double().unsqueeze(1)
        along = torch.sum(dy * w * s, 1, keepdim=True)
        dx = dy * w * r - s * r.pow(3) * along / case["n"]
        if state["dsum"] is not None:
            dx += state["dsum"].double()
        return {"dx": dx, "dweight": torch.sum(dy * s * r, 0)}
    if kind == "product":
        y = torch.mm(state["x"].double(), state["w"].double().t().contiguous())
        return {"y": y * torch.outer(state["x_scales"].double(), state["w_scales"].double())}
    x, label = state["logits"].double(), state["labels"].long()
    lse = torch.logsumexp(x, 1)
    logp = torch.sub(x, lse.unsqueeze(1))
    p = logp.exp()
    entropy = lse - (p * x.clamp(min=-1e4)).sum(1)
    index = torch.arange(case["rows"], device="cuda")
    out = {"logprob": torch.where(label < 0, 0.0, logp[index, label.clamp(min=0)]), "entropy": entropy}
    if kind == "score":
        if case["top"]:
            value, order = x.sort(dim=1, descending=True, stable=True)
            out["top_classes"] = order[:, :case["top"]].int()
            out["top_logprobs"] = value[:, :case["top"]] - lse.unsqueeze(1)
        return out
    chosen = torch.zeros_like(p)
    chosen[index, label.clamp(min=0)] = 1.0
    weight = torch.where(label < 0, 0.0, state["dlogprob"].double()).unsqueeze(1)
    out["dlogits"] = weight * (chosen - p) - state["dentropy"].double().unsqueeze(1) * p * (logp.clamp(min=-1e4) + entropy.unsqueeze(1))
    return out
