"""Speed and results of the operators that train and use a gated block: the block itself and the AdamW step.

The gated block is the predictor Y = (act(X Wg) * (X Wu)) Wd of a mini-batch X (rows x p): forward as a server answers
(also for a single row) or as a training step runs it (keeping G = X Wg and U = X Wu), and backward from dY.  The AdamW
step updates many parameter tensors at once from their gradients, with its moments in 32 bits or in 8.

`own` false: elementary torch operations in 32 bits, rounded once at the end.  `own` true: the framework's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256                 # elements that share a scale where the moments are held in 8 bits
TINY = 2.0 ** -126          # a block whose largest moment is below this is held as zeros


def _gated(name, kind, rows, p, hidden, out, dtype="bf16", act="silu", keep=False):
    case = {"kind": kind, "rows": rows, "p": p, "hidden": hidden, "out": out, "dtype": dtype, "act": act, "keep": keep}
    return case if name is None else {"name": name, **case}


def _adamw(name, tensors, total, grad="bf16", copy="bf16", bits=32):
    case = {"kind": "adamw", "tensors": tensors, "total": total, "grad": grad, "copy": copy, "bits": bits}
    return case if name is None else {"name": name, **case}


def listed():
    return [
        # one row of 512 detector features is answered: a few megabytes of weights, latency is all there is
        _gated("gated_one_row", "forward", rows=1, p=512, hidden=2_048, out=1_000),
        # one wide row: 201 MB of weights stream past it
        _gated("gated_one_row_wide", "forward", rows=1, p=4_096, hidden=8_192, out=4_096, act="gelu"),
        # a handful of rows that arrived together, wide features, 1,000 classes
        _gated("gated_few_rows", "forward", rows=20, p=4_096, hidden=8_192, out=1_000, dtype="f16"),
        # training forward with nothing a multiple of anything
        _gated("gated_forward_ragged", "forward", rows=777, p=123, hidden=1_365, out=130, act="relu", keep=True),
        # training forward of a mini-batch of the fourth configuration (8,192 rows of 4,096 features)
        _gated("gated_forward_large", "forward", rows=8_192, p=4_096, hidden=8_192, out=4_096, keep=True),
        # backward of a small mini-batch
        _gated("gated_backward_small", "backward", rows=100, p=200, hidden=600, out=130),
        # backward of a mini-batch of 1,000 detector features, odd hidden width, f16 under a loss scale
        _gated("gated_backward_medium", "backward", rows=1_000, p=512, hidden=2_731, out=1_000, dtype="f16", act="gelu"),
        # backward of the large mini-batch
        _gated("gated_backward_large", "backward", rows=8_192, p=4_096, hidden=8_192, out=4_096),
        # the step of a small model: latency
        _adamw("adamw_small", tensors=12, total=40_000, grad="f32", copy="none"),
        # many tensors of all sizes in one flat array, so most of them start at odd places
        _adamw("adamw_many_tensors", tensors=160, total=20_000_003),
        # many small tensors with moments in 8 bits
        _adamw("adamw_8bit_ragged", tensors=64, total=1_000_003, grad="f32", copy="f16", bits=8),
        # the three weights of the large block, moments in 8 bits
        _adamw("adamw_8bit_large", tensors=3, total=3 * 4_096 * 8_192, bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["forward", "forward", "backward", "backward", "adamw", "adamw"])
    if kind == "adamw":
        total = _log_int(rng, 10_000, 60_000_000)
        return _adamw(None, tensors=min(_log_int(rng, 1, 300), total // 100), total=total, grad=rng.choice(["bf16", "f16", "f32"]),
                      copy=rng.choice(["bf16", "f16", "none"]), bits=rng.choice([32, 8]))
    case = _gated(None, kind, rows=_log_int(rng, 1, 8_192), p=_log_int(rng, 64, 4_096), hidden=_log_int(rng, 128, 8_192),
                  out=_log_int(rng, 64, 4_096), dtype=rng.choice(["bf16", "bf16", "f16"]),
                  act=rng.choice(["silu", "gelu", "relu"]), keep=kind == "forward" and rng.random() < 0.5)
    if rng.random() < 0.5:                      # widths that suit the machine, as most models have
        for k in ("p", "hidden", "out"):
            case[k] = -(-case[k] // 64) * 64
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _handle(case, state):
    """What a program keeps between calls: the block's handle or the optimizer."""
    if not own:
        return None
    import paper_2312_08728_amd as B
    if case["kind"] != "adamw":
        acts = {"silu": B.BMGD_ACT_SILU, "gelu": B.BMGD_ACT_GELU, "relu": B.BMGD_ACT_RELU}
        return B.GatedBlock(case["p"], case["hidden"], case["out"], case["rows"],
                            dtype=B.BMGD_F16 if case["dtype"] == "f16" else B.BMGD_BF16, activation=acts[case["act"]])
    return B.AdamW(state["thetas"], state["grads"], copies=state["copies"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                   weight_decay=DECAY, state_bits=case["bits"], state=state["moments"], step=state["k"])


def _sizes(case):
    """Sizes of the tensors of an optimizer case: spread over about three decades, at least one element each."""
    rng = random.Random(case["tensors"] * 1_000_003 + case["total"])
    if case["tensors"] * 10 > case["total"] or case["tensors"] < 4:
        part = [1.0] * case["tensors"]
    else:
        part = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(case["tensors"])]
    scale = (case["total"] - case["tensors"]) / sum(part)
    sizes = [1 + int(scale * w) for w in part]
    sizes[-1] += case["total"] - sum(sizes)
    return sizes


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)

    state = {"case": case}
    if case["kind"] != "adamw":
        rows, p, hidden, out, dtype = case["rows"], case["p"], case["hidden"], case["out"], TYPES[case["dtype"]]
        state["x"] = normal(rows, p, dtype=dtype)
        state["wg"] = normal(p, hidden, scale=p ** -0.5, dtype=dtype)
        state["wu"] = normal(p, hidden, scale=p ** -0.5, dtype=dtype)
        state["wd"] = normal(hidden, out, scale=hidden ** -0.5, dtype=dtype)
        new = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        if case["kind"] == "forward":
            state["y"] = new(rows, out)
            state["g"], state["u"] = (new(rows, hidden), new(rows, hidden)) if case["keep"] else (None, None)
        else:
            state["g"], state["u"] = (state["x"].float() @ state["wg"].float()).to(dtype), (state["x"].float() @ state["wu"].float()).to(dtype)
            # the gradient of a mean over the rows, times the loss scale that 16-bit gradients are trained with
            state["dy"] = normal(rows, out, dtype=dtype)
            state["dx"], state["dwg"], state["dwu"], state["dwd"] = new(rows, p), new(p, hidden), new(p, hidden), new(hidden, out)
        state["handle"] = _handle(case, state)
        return state

    # parameters, gradients and moments are pieces of flat arrays; with moments in 8 bits every tensor starts a block of its own
    sizes, unit = _sizes(case), BLOCK if case["bits"] == 8 else 1
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += -(-n // unit) * unit
    index = torch.arange(total, device="cuda")
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    for s, n in zip(starts, sizes):
        used[s:s + n] = True
    pieces = lambda t: [t[s:s + n] for s, n in zip(starts, sizes)]  # noqa: E731
    size_of = 1e-3 * torch.exp(2.0 * torch.sin(index.float() * 1e-3))            # gradients of very different sizes
    state["theta"] = normal(total, scale=0.02) * used
    state["grad"] = (normal(total) * size_of * used).to(TYPES[case["grad"]])
    state["copy"] = torch.zeros(total, dtype=TYPES[case["copy"]], device="cuda") if case["copy"] != "none" else None
    state["thetas"], state["grads"] = pieces(state["theta"]), pieces(state["grad"])
    state["copies"] = pieces(state["copy"]) if state["copy"] is not None else None
    m = normal(total) * size_of * 0.3 * used
    s = (normal(total).square() * 0.2 + 0.8 * torch.rand(total, generator=gen, device="cuda")) * size_of.square() * used
    state["k"] = 100
    if case["bits"] == 32:
        state["m"], state["s"] = m, s
        state["moments"] = list(zip(pieces(m), pieces(s)))
    else:
        state["mc"], state["ma"] = _coded_m(m)
        state["sc"], state["sa"] = _coded_s(s)
        blocks = [(b // BLOCK, -(-n // BLOCK)) for b, n in zip(starts, sizes)]
        of_blocks = lambda t: [t[b:b + n] for b, n in blocks]  # noqa: E731
        state["moments"] = list(zip(pieces(state["mc"]), pieces(state["sc"]), of_blocks(state["ma"]), of_blocks(state["sa"])))
        state["m"], state["s"] = torch.zeros_like(m), torch.zeros_like(s)
        state["values"] = list(zip(pieces(state["m"]), pieces(state["s"])))
    state["handle"] = _handle(case, state)
    return state


# ---- the plain forms --------------------------------------------------------------------------------------------------
def _act(g, act):
    """act(g) and its derivative."""
    if act == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    cdf = 0.5 * (1.0 + torch.erf(g * 0.5 ** 0.5))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5


def _forward(case, x, wg, wu, wd):
    g, u = x @ wg, x @ wu
    y = (_act(g, case["act"])[0] * u) @ wd
    return {"y": y, "g": g, "u": u} if case["keep"] else {"y": y}


def _backward(case, dy, x, wg, wu, wd, g, u):
    a, da = _act(g, case["act"])
    dh = dy @ wd.t()
    du, dg = dh * a, dh * u * da
    return {"dx": dg @ wg.t() + du @ wu.t(), "dwg": x.t() @ dg, "dwu": x.t() @ du, "dwd": (a * u).t() @ dy}


def _coded_m(m):
    """8-bit codes and scales of first moments: m = scale * sgn(code) * (code / 127)^2, scale = the block's largest |m|."""
    size = m.view(-1, BLOCK).abs()
    top = size.amax(1)
    top = torch.where(top >= TINY, top, torch.zeros_like(top))
    inv = torch.where(top > 0, 1.0 / top, torch.zeros_like(top))
    code = torch.round(127.0 * torch.sqrt(size * inv[:, None])) * torch.sign(m.view(-1, BLOCK))
    return code.to(torch.int8).view(-1), top


def _coded_s(s):
    """8-bit codes and scales of second moments: s = scale * (code / 255)^4; what is not zero keeps a code of at least 1."""
    s = s.view(-1, BLOCK)
    top = s.amax(1)
    top = torch.where(top >= TINY, top, torch.zeros_like(top))
    inv = torch.where(top > 0, 1.0 / top, torch.zeros_like(top))
    code = torch.round(255.0 * torch.sqrt(torch.sqrt(s * inv[:, None])))
    code = torch.where((s > 0) & (top[:, None] > 0), torch.clamp(code, min=1.0), code)
    return code.to(torch.uint8).view(-1), top


def _value_m(code, top):
    t = code.float() * (1.0 / 127.0)
    return (top[:, None] * (t * t.abs()).view(-1, BLOCK)).view(-1)


def _value_s(code, top):
    t = code.float() * (1.0 / 255.0)
    t = t * t
    return (top[:, None] * (t * t).view(-1, BLOCK)).view(-1)


def _step(theta, g, m, s, k):
    m = BETA1 * m + (1.0 - BETA1) * g
    s = BETA2 * s + (1.0 - BETA2) * (g * g)
    top = m * (1.0 / (1.0 - BETA1 ** k))
    bottom = torch.sqrt(s * (1.0 / (1.0 - BETA2 ** k))) + EPS
    return theta * (1.0 - LR * DECAY) - LR * (top / bottom), m, s


def _plain_adamw(state):
    state["k"] += 1
    if state["case"]["bits"] == 32:
        theta, m, s = _step(state["theta"], state["grad"].float(), state["m"], state["s"], state["k"])
        state["m"].copy_(m)
        state["s"].copy_(s)
    else:
        m, s = _value_m(state["mc"], state["ma"]), _value_s(state["sc"], state["sa"])
        theta, m, s = _step(state["theta"], state["grad"].float(), m, s, state["k"])
        for to, value in zip((state["mc"], state["ma"], state["sc"], state["sa"]), _coded_m(m) + _coded_s(s)):
            to.copy_(value)
        state["m"].copy_(_value_m(state["mc"], state["ma"]))
        state["s"].copy_(_value_s(state["sc"], state["sa"]))
    state["theta"].copy_(theta)
    if state["copy"] is not None:
        state["copy"].copy_(theta)


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(state):
    case, handle = state["case"], state["handle"]
    if case["kind"] == "adamw":
        if own:
            handle.step()
            if case["bits"] == 8:
                handle.moments(out=state["values"])      # what the 8 bits stand for, as a program saves them
        else:
            _plain_adamw(state)
        out = {"theta": state["theta"], "m": state["m"], "s": state["s"]}
        return out if state["copy"] is None else {**out, "copy": state["copy"]}
    x, weights = state["x"], (state["wg"], state["wu"], state["wd"])
    if case["kind"] == "forward":
        if own:
            handle.forward(x, *weights, state["y"], g=state["g"], u=state["u"])
            return {"y": state["y"], "g": state["g"], "u": state["u"]} if case["keep"] else {"y": state["y"]}
        out = _forward(case, *(t.float() for t in (x, *weights)))
    else:
        if own:
            handle.backward(state["dy"], x, *weights, state["g"], state["u"], state["dx"], state["dwg"], state["dwu"], state["dwd"])
            return {k: state[k] for k in ("dx", "dwg", "dwu", "dwd")}
        out = _backward(case, *(t.float() for t in (state["dy"], x, *weights, state["g"], state["u"])))
    return {k: v.to(TYPES[case["dtype"]]) for k, v in out.items()}


def work(case):
    """Each input read once and each output written once.  Moments in 8 bits: the step (codes in and out) and then the
    values that the codes stand for (codes in, 32 bits out)."""
    if case["kind"] == "adamw":
        item = {"f32": 4, "bf16": 2, "f16": 2, "none": 0}
        each = 8 + item[case["grad"]] + item[case["copy"]] + (16 if case["bits"] == 32 else 4 + 10)
        return {"bytes": each * case["total"], "flops": 20 * case["total"]}
    r, p, f, c = case["rows"], case["p"], case["hidden"], case["out"]
    if case["kind"] == "forward":
        return {"bytes": 2 * (r * p + 2 * p * f + f * c + r * c + (2 * r * f if case["keep"] else 0)), "flops": 2 * r * f * (2 * p + c)}
    return {"bytes": 2 * (2 * r * p + 4 * p * f + 2 * f * c + r * c + 2 * r * f), "flops": 4 * r * f * (2 * p + c)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(state)
    x, wg, wu, wd = (state[k].double() for k in ("x", "wg", "wu", "wd"))
    if case["kind"] == "forward":
        g, u = x.mm(wg), x.mm(wu)
        y = (_exact_act(g, case["act"])[0] * u).mm(wd)
        return {"y": y, "g": g, "u": u} if case["keep"] else {"y": y}
    g, u, dy = (state[k].double() for k in ("g", "u", "dy"))
    value, slope = _exact_act(g, case["act"])
    dh = torch.mm(dy, wd.t().contiguous())
    dg, du = dh * slope * u, dh * value
    dx = torch.mm(torch.cat([dg, du], 1), torch.cat([wg, wu], 1).t().contiguous())
    xt = x.t().contiguous()
    return {"dx": dx, "dwg": xt.mm(dg), "dwu": xt.mm(du), "dwd": (value * u).t().contiguous().mm(dy)}


def _exact_act(g, act):
    if act == "relu":
        return torch.clamp(g, min=0.0), torch.where(g > 0, torch.ones_like(g), torch.zeros_like(g))
    if act == "silu":
        sig = torch.sigmoid(g)
        return g * sig, sig + g * sig * (1.0 - sig)
    phi = torch.exp(-g.square() / 2.0) / math.sqrt(2.0 * math.pi)
    big_phi = torch.special.ndtr(g)
    return g * big_phi, big_phi + g * phi


def _exact_adamw(state):
    case, k = state["case"], state["k"] + 1
    g, theta = state["grad"].double(), state["theta"].double()
    if case["bits"] == 8:
        t, v = state["mc"].double() / 127.0, state["sc"].double() / 255.0
        m = t.abs() * t * state["ma"].double().repeat_interleave(BLOCK)
        s = v.pow(4) * state["sa"].double().repeat_interleave(BLOCK)
    else:
        m, s = state["m"].double(), state["s"].double()
    m = BETA1 * m + (1.0 - BETA1) * g
    s = BETA2 * s + (1.0 - BETA2) * g.square()
    rate = LR / (1.0 - BETA1 ** k)
    theta = theta - LR * DECAY * theta - rate * m / ((s / (1.0 - BETA2 ** k)).sqrt() + EPS)
    if case["bits"] == 8:
        a = m.abs().view(-1, BLOCK).max(1, keepdim=True).values
        b = s.view(-1, BLOCK).max(1, keepdim=True).values
        q = torch.round(127.0 * (m.abs().view(-1, BLOCK) / a.clamp(min=1e-300)).sqrt())
        m = (a * (q / 127.0).square() * torch.sign(m.view(-1, BLOCK))).view(-1)
        q = torch.round(255.0 * (s.view(-1, BLOCK) / b.clamp(min=1e-300)).pow(0.25))
        q = torch.maximum(q, (s.view(-1, BLOCK) > 0).double())
        s = (b * (q / 255.0).pow(4)).view(-1)
    out = {"theta": theta, "m": m, "s": s}
    return out if state["copy"] is None else {**out, "copy": theta}
