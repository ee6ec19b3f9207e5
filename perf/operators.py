"""Cases of the client's training operators: linear layers and 8-bit activation checkpoints.

A sender of EDEN trains before it sends.  Its step is a feed-forward block: matrix products
with bias, activation and residual in the epilogue (``linear``), activations kept for the
backward pass in 8 bits (``checkpoint``), and the three products of the backward pass that
read those checkpoints (``act_backward``, ``input_grad``, ``weight_grad``).  The weight
gradient is fp32 and is what ``eden_encode`` takes as the client's vector.

The 8-bit form: rows of features are cut into groups of 32 (the last one of a row may be
shorter); a group keeps one power of two 2^e, the smallest with max|v| <= 127 * 2^e, and one
code per value, v / 2^e rounded to the nearest whole number, ties to even.  Codes are int8
[rows, features]; the exponents are uint8 [rows, ceil(features / 32)], e + 127, at least 1,
and 255 where a group holds an infinity or a NaN (its values are then NaN).

``run`` computes the operators from elementary torch operations where ``own`` is false and
calls the framework where it is true.
"""
import math

import torch

own = False

GROUP = 32
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token answered by the current model: a 2^24-coordinate weight read once, latency counts
        {"name": "linear-token", "op": "linear", "m": 1, "n": 4096, "k": 4096, "dtype": "bf16", "act": "silu", "residual": True, "save": "none"},
        # a few sequences evaluated together on a layer whose sizes fit no tile, unaligned rows
        {"name": "linear-ragged-batch", "op": "linear", "m": 13, "n": 2731, "k": 1000, "dtype": "fp16", "act": "relu", "residual": True, "save": "none"},
        # forward of a training step: up projection that keeps its pre-activation in 8 bits
        {"name": "linear-train-save", "op": "linear", "m": 4096, "n": 4096, "k": 1024, "dtype": "bf16", "act": "gelu", "residual": False, "save": "pre"},
        # the widest layer (2^26 weights) over a whole batch of sequences
        {"name": "linear-train-large", "op": "linear", "m": 8192, "n": 16384, "k": 4096, "dtype": "bf16", "act": "gelu_tanh", "residual": False, "save": "none"},
        # a small activation saved and restored: latency counts, last group of each row is short
        {"name": "checkpoint-small", "op": "checkpoint", "m": 61, "n": 1001, "dtype": "fp16"},
        # a block's activations over a whole batch
        {"name": "checkpoint-large", "op": "checkpoint", "m": 16384, "n": 4096, "dtype": "bf16"},
        # activation gradient of a small, unaligned layer
        {"name": "act-backward-ragged", "op": "act_backward", "m": 333, "n": 2731, "dtype": "fp16", "act": "silu"},
        # activation gradient and bias gradient of the widest layer
        {"name": "act-backward-large", "op": "act_backward", "m": 8192, "n": 16384, "dtype": "bf16", "act": "gelu"},
        # backward through an odd layer and the activation before it, in one pass
        {"name": "input-grad-ragged", "op": "input_grad", "m": 1999, "n": 1000, "k": 2731, "dtype": "fp16", "act": "relu", "residual": False, "pre": True},
        # backward through a square layer whose input also feeds a residual branch
        {"name": "input-grad-residual", "op": "input_grad", "m": 8192, "n": 4096, "k": 4096, "dtype": "bf16", "act": "none", "residual": True, "pre": False},
        # weight gradient of 2^20 coordinates over a few sequences: few output tiles, long sum
        {"name": "weight-grad-2e20", "op": "weight_grad", "m": 4096, "n": 1024, "k": 1024, "dtype": "bf16"},
        # weight gradient of 2^24 coordinates over a batch whose token count fits no tile
        {"name": "weight-grad-2e24", "op": "weight_grad", "m": 8191, "n": 4096, "k": 4096, "dtype": "bf16"},
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; two of five are rounded to a multiple of 64 where that fits."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.4 and v >= 64:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(("linear", "linear", "checkpoint", "act_backward", "input_grad", "weight_grad"))
    dtype = rng.choice(("bf16", "fp16"))
    most = 8192 * 16384 * 4096
    while True:
        m, n, k = _size(rng, 1, 8192), _size(rng, 64, 16384), _size(rng, 64, 16384)
        if m * n * k <= most and m * max(n, k) <= 8192 * 16384:
            break
    case = {"op": op, "m": m, "n": n, "dtype": dtype}
    if op == "linear":
        case.update(k=k, act=rng.choice(ACTS), residual=rng.random() < 0.5, save=rng.choice(("none", "pre", "out")))
    elif op == "act_backward":
        case.update(act=rng.choice(ACTS))
    elif op == "input_grad":
        pre = rng.random() < 0.5
        case.update(k=k, act=rng.choice(ACTS) if pre else "none", residual=rng.random() < 0.5 and not pre, pre=pre)
    elif op == "weight_grad":
        case.update(k=k)
    return case


def work(case):
    m, n, k = case["m"], case["n"], case.get("k", 0)
    groups = lambda c: -(-c // GROUP)  # noqa: E731
    if case["op"] == "linear":
        b = 2 * (m * k + n * k + n + m * n * (2 if case["residual"] else 1))
        b += m * (n + groups(n)) if case["save"] != "none" else 0
        return {"bytes": b, "flops": 2 * m * n * k}
    if case["op"] == "checkpoint":  # read and coded, then read back and restored
        return {"bytes": m * (2 * n + 2 * (n + groups(n)) + 2 * n), "flops": 4 * m * n}
    if case["op"] == "act_backward":
        return {"bytes": m * (2 * n + n + groups(n) + 2 * n) + 4 * n, "flops": 20 * m * n}
    if case["op"] == "input_grad":
        b = 2 * (m * n + n * k + m * k * (2 if case["residual"] else 1))
        b += m * (k + groups(k)) + 4 * k if case["pre"] else 0
        return {"bytes": b, "flops": 2 * m * n * k}
    return {"bytes": 2 * m * n + m * (k + groups(k)) + 4 * n * k, "flops": 2 * m * n * k}


# ------------------------------------------------------------------------------------ inputs
def _gauss(g, dtype, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _laplace(g, dtype, *shape, std):
    """Gradients are heavy-tailed: Laplace, as in the synthetic client vectors."""
    u = torch.rand(shape, generator=g, device="cuda") - 0.5
    return (torch.sign(u) * -torch.log1p(-2 * u.abs()).clamp_(max=20.0) * (std / math.sqrt(2.0))).to(dtype)


def _context(nbytes):
    """One context per program, with a workspace for the largest call so far."""
    from paper_2108_08842_b200 import eden

    if _context.held is None or _context.held.workspace_bytes < nbytes:
        _context.held = eden.Context(0, workspace_bytes_=max(nbytes, 1 << 20))
    return _context.held


_context.held = None


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, n, k, t = case["m"], case["n"], case.get("k", 0), TYPES[case["dtype"]]
    s = {"case": case, "type": t}
    op = case["op"]
    if op == "linear":
        s["x"] = _gauss(g, t, m, k)
        s["weight"] = _gauss(g, t, n, k, std=k ** -0.5)
        s["bias"] = _gauss(g, t, n, std=0.1)
        s["residual"] = _gauss(g, t, m, n) if case["residual"] else None
        s["out"] = torch.empty((m, n), dtype=t, device="cuda")
    elif op == "checkpoint":
        # activations of a block: features of unequal scale
        s["x"] = (torch.randn((m, n), generator=g, device="cuda") * torch.exp(0.5 * torch.randn(n, generator=g, device="cuda"))).to(t)
        s["out"] = torch.empty((m, n), dtype=t, device="cuda")
    elif op == "act_backward":
        s["dy"] = _laplace(g, t, m, n, std=0.02)
        s["pre"] = _code(torch.randn((m, n), generator=g, device="cuda"))
        s["out"] = torch.empty((m, n), dtype=t, device="cuda")
        s["bias_grad"] = torch.empty(n, dtype=torch.float32, device="cuda")
    elif op == "input_grad":
        s["dz"] = _laplace(g, t, m, n, std=0.02)
        s["weight"] = _gauss(g, t, n, k, std=k ** -0.5)
        s["residual"] = _laplace(g, t, m, k, std=0.02) if case["residual"] else None
        s["pre"] = _code(torch.randn((m, k), generator=g, device="cuda")) if case["pre"] else None
        s["out"] = torch.empty((m, k), dtype=t, device="cuda")
        s["bias_grad"] = torch.empty(k, dtype=torch.float32, device="cuda") if case["pre"] else None
    else:
        s["dz"] = _laplace(g, t, m, n, std=0.02)
        s["saved"] = _code(torch.randn((m, k), generator=g, device="cuda").to(t))
        s["out"] = torch.empty((n, k), dtype=torch.float32, device="cuda")
    if own:  # the handle and the workspace that a program keeps
        from paper_2108_08842_b200 import eden

        s["ctx"] = _context(eden.linear_workspace_bytes(m, n, max(k, 1)))
    return s


# ------------------------------------------------------------------------------------ plain forms
def _code(v):
    """8-bit form of v [rows, features]: (int8 codes, uint8 exponents)."""
    m, n = v.shape
    pad = -n % GROUP
    v = torch.nn.functional.pad(v.float(), (0, pad)).view(m, (n + pad) // GROUP, GROUP)
    bits = v.abs().amax(dim=2).contiguous().view(torch.int32)
    # max = 1.f * 2^E needs 2^(E - 6), or 2^(E - 5) where 1.f is over 127 / 64
    e = ((bits + 0x1FFFF) >> 23) - 6
    e = torch.where(bits >= 0x7F800000, 255, e.clamp(min=1))
    step = ((254 - e.clamp(max=253)) << 23).view(torch.float32)
    codes = torch.where(e[:, :, None] == 255, 0.0, torch.round(v * step[:, :, None]))
    return codes.to(torch.int8).view(m, n + pad)[:, :n].contiguous(), e.to(torch.uint8)


def _value(codes, exps):
    """The values, in 32 bits, that an 8-bit form stands for."""
    n = codes.shape[1]
    scale = (exps.to(torch.int32) << 23).view(torch.float32)
    return codes.float() * scale.repeat_interleave(GROUP, dim=1)[:, :n]


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_plain(s):
    case, t = s["case"], s["type"]
    op = case["op"]
    if op == "linear":
        z = s["x"].float() @ s["weight"].float().t() + s["bias"].float()
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        y = y.to(t)
        if case["save"] == "none":
            return {"y": y}
        return {"y": y, "saved": _value(*_code(z if case["save"] == "pre" else y)).to(t)}
    if op == "checkpoint":
        return {"x": _value(*_code(s["x"])).to(t)}
    if op == "act_backward":
        dz = s["dy"].float() * _act_slope(_value(*s["pre"]), case["act"])
        return {"dz": dz.to(t), "bias_grad": dz.sum(dim=0)}
    if op == "input_grad":
        dx = s["dz"].float() @ s["weight"].float()
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        if s["pre"] is None:
            return {"dx": dx.to(t)}
        dx = dx * _act_slope(_value(*s["pre"]), case["act"])
        return {"dx": dx.to(t), "bias_grad": dx.sum(dim=0)}
    return {"weight_grad": s["dz"].float().t() @ _value(*s["saved"])}


def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    op = case["op"]
    if op == "linear":
        if case["save"] == "none":
            return {"y": ctx.linear(s["x"], s["weight"], s["bias"], act=case["act"], residual=s["residual"], out=s["out"])}
        y, saved = ctx.linear(s["x"], s["weight"], s["bias"], act=case["act"], residual=s["residual"], out=s["out"], save=case["save"])
        return {"y": y, "saved": ctx.checkpoint_restore(saved, s["type"])}
    if op == "checkpoint":
        return {"x": ctx.checkpoint_restore(ctx.checkpoint_save(s["x"]), s["type"], out=s["out"])}
    if op == "act_backward":
        dz, db = ctx.act_backward(s["dy"], s["pre"], act=case["act"], out=s["out"], bias_grad=s["bias_grad"])
        return {"dz": dz, "bias_grad": db}
    if op == "input_grad":
        if s["pre"] is None:
            return {"dx": ctx.linear_input_grad(s["dz"], s["weight"], residual=s["residual"], out=s["out"])}
        dx, db = ctx.linear_input_grad(s["dz"], s["weight"], pre=s["pre"], act=case["act"], out=s["out"], bias_grad=s["bias_grad"])
        return {"dx": dx, "bias_grad": db}
    return {"weight_grad": ctx.linear_weight_grad(s["dz"], s["saved"], out=s["out"])}


# ------------------------------------------------------------------------------------ 64 bits
def _exact_coded(v, dtype):
    """What the 8-bit form of v stands for, from the definition: the least whole e with
    max <= 127 * 2^e in each group, values rounded to multiples of 2^e."""
    short = -v.shape[1] % GROUP
    part = torch.cat([v, v.new_zeros(v.shape[0], short)], dim=1).unflatten(1, (-1, GROUP))
    mant, expo = torch.frexp(part.abs().amax(dim=2, keepdim=True) / 127)  # mant * 2^expo with 0.5 <= mant < 1
    expo = torch.where(mant == 0.5, expo - 1, expo).clamp(min=-126)
    unit = torch.ldexp(torch.ones_like(mant), expo)
    return (torch.round(part / unit) * unit).flatten(1)[:, : v.shape[1]].to(dtype)


def _exact_held(saved):
    codes, exps = saved
    column = torch.arange(codes.shape[1], device=codes.device) // GROUP
    return torch.ldexp(codes.double(), exps[:, column].to(torch.int32) - 127)


def _exact_act(z, act):
    z = z.detach().requires_grad_(True)
    with torch.enable_grad():
        y = {
            "none": lambda: z * 1.0,
            "relu": lambda: z.clamp(min=0),
            "gelu": lambda: z * 0.5 * torch.special.erfc(-z / 2 ** 0.5),
            "gelu_tanh": lambda: z * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)),
            "silu": lambda: z * torch.sigmoid(z),
        }[act]()
    return y, z


def _exact_slope(z, act):
    y, z = _exact_act(z, act)
    if act == "relu":
        return torch.heaviside(z.detach(), torch.zeros_like(z))
    return torch.autograd.grad(y.sum(), z)[0]


def exact(case, seed):
    s, t = prepare(case, seed), TYPES[case["dtype"]]
    op = case["op"]
    if op == "linear":
        z = torch.addmm(s["bias"].double(), s["x"].double(), s["weight"].double().t())
        if case["save"] == "pre":
            saved = _exact_coded(z, t)
        y = _exact_act(z, case["act"])[0].detach()
        del z
        if case["residual"]:
            y += s["residual"].double()
        if case["save"] == "none":
            return {"y": y}
        return {"y": y, "saved": saved if case["save"] == "pre" else _exact_coded(y.to(t).double(), t)}
    if op == "checkpoint":
        return {"x": _exact_coded(s["x"].double(), t)}
    if op == "act_backward":
        dz = s["dy"].double() * _exact_slope(_exact_held(s["pre"]), case["act"])
        return {"dz": dz, "bias_grad": dz.sum(dim=0)}
    if op == "input_grad":
        dx = torch.mm(s["dz"].double(), s["weight"].double())
        if case["residual"]:
            dx += s["residual"].double()
        if not case["pre"]:
            return {"dx": dx}
        dx *= _exact_slope(_exact_held(s["pre"]), case["act"])
        return {"dx": dx, "bias_grad": dx.sum(dim=0)}
    return {"weight_grad": torch.mm(s["dz"].double().t(), _exact_held(s["saved"]))}
