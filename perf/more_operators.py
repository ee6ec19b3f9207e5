"""Cases of the operators around and inside a client's feed-forward blocks: what joins a block to
the residual stream, and products in microscaled 4-bit floating point.

    join           x = scale * residual + gate * dropout(after(h)),  y = before(x)
                   after: the norm behind a block, before: the norm in front of the next one
    join_backward  its gradients, from dx and dy
    dropout        scale * residual + dropout(x), the mask from a counter-based generator, not stored
    mx4_quantize   a matrix in groups of 32 values of 4 bits with a power of two each, along its
                   rows and along its columns (the two forms that a training step's products read)
    mx4_linear     act(x W^T + bias) + residual with both operands in that form
    mx4_backward   the backward products of such a layer: dz is quantised both ways, then
                   dx = (dz W) * act'(z) with its column sums, and dW = dz^T x in 32 bits

Norms: "rms" is v / sqrt(mean(v^2) + eps) * weight + bias; "layer" takes the mean off first, and
divides by the deviation sqrt(mean((v - mean)^2) + eps).  Their statistics are the mean (0 for
"rms") and one over the divisor.

Dropout: value (row, col) has number col % 8 of the eight 16-bit halves (word by word, the low half
first) of Philox4x32-10 with counter (col // 8, row, 3, 0) and the 64-bit seed as its key.  It is kept
where the number is below round(65536 * (1 - drop)), and divided by the exact chance of that.

4-bit groups: a group of 32 along the sum's axis keeps 2^e, the smallest with max|v| <= 6 * 2^e (e
at least -126), and per value sign and magnitude out of 0, 0.5, 1, 1.5, 2, 3, 4, 6 of v / 2^e,
rounded to nearest, ties to the even code.

``run`` computes the operators from elementary torch operations where ``own`` is false and
calls the framework where it is true.
"""
import math

import numpy as np
import torch

own = False

GROUP = 32
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS = 1e-6


# ------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token between two blocks of the current model: latency counts
        {"name": "join-token", "op": "join", "m": 1, "n": 4096, "dtype": "bf16", "after": "rms", "before": "rms", "gate": "vector", "residual": True, "drop": 0.0, "bias": False, "train": False},
        # a training batch between two blocks: both norms, the gate and dropout in one pass
        {"name": "join-train-large", "op": "join", "m": 16384, "n": 4096, "dtype": "bf16", "after": "rms", "before": "rms", "gate": "vector", "residual": True, "drop": 0.1, "bias": False, "train": True},
        # backward of a small step on a width that fits no tile, unaligned rows, a gate per value
        {"name": "join-backward-ragged", "op": "join_backward", "m": 333, "n": 2731, "dtype": "fp16", "after": "layer", "before": "layer", "gate": "matrix", "residual": True, "drop": 0.2, "bias": True, "held": False},
        # backward of the training batch, from activations that were kept in 8 bits
        {"name": "join-backward-large", "op": "join_backward", "m": 16384, "n": 4096, "dtype": "bf16", "after": "rms", "before": "rms", "gate": "vector", "residual": True, "drop": 0.1, "bias": False, "held": True},
        # dropout of a few sequences on unaligned rows: latency counts
        {"name": "dropout-small", "op": "dropout", "m": 61, "n": 1001, "dtype": "fp16", "drop": 0.5, "residual": False},
        # dropout of a block's result on its way into the residual stream, a whole batch
        {"name": "dropout-large", "op": "dropout", "m": 16384, "n": 4096, "dtype": "bf16", "drop": 0.1, "residual": True},
        # a small gradient quantised both ways, the last group of each row and column is short
        {"name": "mx4-quantize-ragged", "op": "mx4_quantize", "m": 333, "n": 2731, "dtype": "fp16"},
        # the gradient of a wide layer quantised both ways
        {"name": "mx4-quantize-large", "op": "mx4_quantize", "m": 8192, "n": 8192, "dtype": "bf16"},
        # one token answered by a model whose 2^24-coordinate weights are kept in 4 bits
        {"name": "mx4-linear-token", "op": "mx4_linear", "m": 1, "n": 4096, "k": 4096, "dtype": "bf16", "act": "silu", "residual": True},
        # the widest layer (2^26 weights) over a whole batch of sequences
        {"name": "mx4-linear-large", "op": "mx4_linear", "m": 8192, "n": 16384, "k": 4096, "dtype": "bf16", "act": "gelu_tanh", "residual": False},
        # backward of an odd layer over an odd batch
        {"name": "mx4-backward-ragged", "op": "mx4_backward", "m": 1999, "n": 1000, "k": 2731, "dtype": "fp16", "act": "relu"},
        # backward of a square layer of 2^24 weights over a batch whose token count fits no tile
        {"name": "mx4-backward-large", "op": "mx4_backward", "m": 8191, "n": 4096, "k": 4096, "dtype": "bf16", "act": "gelu"},
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm; two of five are rounded to a multiple of 64 where that fits."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.4 and v >= 64:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(("join", "join", "join_backward", "join_backward", "dropout", "mx4_quantize", "mx4_linear", "mx4_linear", "mx4_backward"))
    dtype = rng.choice(("bf16", "fp16"))
    if op in ("join", "join_backward", "dropout", "mx4_quantize"):
        while True:
            m, n = _size(rng, 1, 16384), _size(rng, 64, 16384)
            if m * n <= 16384 * 4096:
                break
        case = {"op": op, "m": m, "n": n, "dtype": dtype}
        if op == "mx4_quantize":
            return case
        drop = rng.choice((0.0, 0.1, 0.25, 0.5, rng.uniform(0.01, 0.9)))
        if op == "dropout":
            case.update(drop=drop, residual=rng.random() < 0.5)
            return case
        after, before = rng.choice((("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "none"), ("none", "layer"), ("layer", "rms")))
        case.update(after=after, before=before, gate=rng.choice(("none", "vector", "matrix")), residual=rng.random() < 0.8, drop=drop, bias=rng.random() < 0.5)
        case.update(train=rng.random() < 0.5) if op == "join" else case.update(held=rng.random() < 0.5)
        return case
    most = 8191 * 4096 * 4096 if op == "mx4_backward" else 8192 * 16384 * 4096
    while True:
        m, n, k = _size(rng, 1, 8192), _size(rng, 64, 16384), _size(rng, 64, 16384)
        if m * n * k <= most and m * max(n, k) <= (8192 * 16384 if op == "mx4_linear" else 8191 * 4096):
            break
    case = {"op": op, "m": m, "n": n, "k": k, "dtype": dtype, "act": rng.choice(ACTS)}
    if op == "mx4_linear":
        case.update(residual=rng.random() < 0.5)
    return case


def _groups(c):
    return -(-c // GROUP)


def _mx4_bytes(rows, cols):
    """16 bytes of codes and one of exponent for each group of a row."""
    return rows * _groups(cols) * 17


def work(case):
    m, n, k = case["m"], case["n"], case.get("k", 0)
    if case["op"] == "join":
        matrices = 2 + int(case["residual"]) + int(case["before"] != "none") + int(case["gate"] == "matrix")   # h, x; residual, y, gate
        norms = [kind for kind in (case["after"], case["before"]) if kind != "none"]
        vectors = len(norms) * (1 + int(case["bias"])) + int(case["gate"] == "vector")
        return {"bytes": 2 * m * n * matrices + 2 * n * vectors + (8 * m * len(norms) if case["train"] else 0), "flops": m * n * (12 + (40 if case["drop"] else 0))}
    if case["op"] == "join_backward":
        pre, post = int(case["before"] != "none"), int(case["after"] != "none")
        needs_h = bool(post) or case["gate"] != "none"
        each = (1 + 1 / GROUP) if case["held"] else 2
        b = 2 * m * n * (2 + pre + int(case["residual"]))                                # dx, dh, dy, d residual
        b += m * n * each * (pre + int(needs_h)) + (4 * m * n if case["gate"] == "matrix" else 0)
        b += 8 * m * (pre + post) + n * (6 * (pre + post) + (4 * (pre + post) if case["bias"] else 0) + (6 if case["gate"] == "vector" else 0))
        return {"bytes": int(b), "flops": m * n * (30 + (40 if case["drop"] else 0))}
    if case["op"] == "dropout":
        return {"bytes": 2 * m * n * (3 if case["residual"] else 2), "flops": 45 * m * n}
    if case["op"] == "mx4_quantize":   # read once, both forms written; what they stand for is read back and restored
        return {"bytes": 2 * m * n + 2 * (_mx4_bytes(m, n) + _mx4_bytes(n, m)) + 4 * m * n, "flops": 8 * m * n}
    if case["op"] == "mx4_linear":
        return {"bytes": 2 * m * k + _mx4_bytes(n, k) + 2 * n + 2 * m * n * (2 if case["residual"] else 1), "flops": 2 * m * n * k}
    pre = m * (k + _groups(k)) if case["act"] != "none" else 0
    return {"bytes": 2 * m * n + _mx4_bytes(k, n) + _mx4_bytes(k, m) + pre + 2 * m * k + 4 * k + 4 * n * k, "flops": 4 * m * n * k}


# ------------------------------------------------------------------------------------ inputs
def _gauss(g, dtype, *shape, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


def _laplace(g, dtype, *shape, std):
    """Gradients are heavy-tailed: Laplace, as in the synthetic client vectors."""
    u = torch.rand(shape, generator=g, device="cuda") - 0.5
    return (torch.sign(u) * (-torch.log1p(-2 * u.abs())).clamp_(max=20.0) * (std / math.sqrt(2.0))).to(dtype)   # u = -0.5 stays finite


def _features(g, dtype, m, n):
    """Activations of a block: features of unequal scale and a mean of their own."""
    scale = torch.exp(0.5 * torch.randn(n, generator=g, device="cuda"))
    return (torch.randn((m, n), generator=g, device="cuda") * scale + 0.3 * torch.randn(n, generator=g, device="cuda")).to(dtype)


def _context(nbytes):
    """One context per program, with a workspace for the largest call so far."""
    from paper_2108_08842_b200 import eden

    if _context.held is None or _context.held.workspace_bytes < nbytes:
        _context.held = eden.Context(0, workspace_bytes_=max(nbytes, 1 << 20))
    return _context.held


_context.held = None


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, n, k, t, op = case["m"], case["n"], case.get("k", 0), TYPES[case["dtype"]], case["op"]
    s = {"case": case, "type": t, "seed": (seed * 0x9E3779B97F4A7C15 + 12345) % 2 ** 64}
    if op in ("join", "join_backward"):
        s["h"] = _features(g, t, m, n)
        s["residual"] = _features(g, t, m, n) if case["residual"] else None
        s["gate"] = {"none": lambda: None, "vector": lambda: _gauss(g, t, n, std=0.2, mean=0.5), "matrix": lambda: _gauss(g, t, m, n, std=0.2, mean=0.5)}[case["gate"]]()
        for side in ("after", "before"):
            weight, bias = _gauss(g, t, n, std=0.1, mean=1.0), _gauss(g, t, n, std=0.1)
            s[side] = None if case[side] == "none" else (case[side], weight, bias if case["bias"] else None)
        s["scale"] = 0.75 if case["residual"] else 0.0
    if op == "join":
        s["out"] = torch.empty((m, n), dtype=t, device="cuda"), torch.empty((m, n), dtype=t, device="cuda") if s["before"] else None
    elif op == "join_backward":
        # the join's result is on hand from the forward pass, as are both norms' statistics
        s["x"] = _features(g, t, m, n)
        s["dx"], s["dy"] = _laplace(g, t, m, n, std=0.02), _laplace(g, t, m, n, std=0.02) if s["before"] else None
        s["after_stats"] = _statistics(s["h"].float(), case["after"]) if s["after"] else None
        s["before_stats"] = _statistics(s["x"].float(), case["before"]) if s["before"] else None
        if not (s["after"] or case["gate"] != "none"):
            s["h"] = None                                  # nothing depends on it
        if not s["before"]:
            s["x"] = None
        for name in ("h", "x"):
            if case["held"] and s[name] is not None:
                s[name] = _code8(s[name])
        s["residual"] = None
    elif op == "dropout":
        s["x"] = _features(g, t, m, n)
        s["residual"] = _gauss(g, t, m, n) if case["residual"] else None
        s["out"] = torch.empty((m, n), dtype=t, device="cuda")
    elif op == "mx4_quantize":
        s["x"] = _laplace(g, t, m, n, std=0.02)
    elif op == "mx4_linear":
        s["x"], weight = _gauss(g, t, m, k), _gauss(g, t, n, k, std=k ** -0.5)
        s["bias"], s["residual"] = _gauss(g, t, n, std=0.1), _gauss(g, t, m, n) if case["residual"] else None
        s["out"] = torch.empty((m, n), dtype=t, device="cuda")
    else:
        s["dz"] = _laplace(g, t, m, n, std=0.02)
        weight, x = _gauss(g, t, n, k, std=k ** -0.5), _gauss(g, t, m, k)
        s["pre"] = _code8(torch.randn((m, k), generator=g, device="cuda"))
        s["out"], s["bias_grad"] = torch.empty((m, k), dtype=t, device="cuda"), torch.empty(k, device="cuda")
        s["weight_grad"] = torch.empty((n, k), device="cuda")
    if own:  # the handle and the workspace that a program keeps, and what it keeps in 4 bits
        from paper_2108_08842_b200 import eden

        ctx = s["ctx"] = _context(max(eden.block_workspace_bytes(n), eden.mx4_workspace_bytes(m, n, max(k, 1))))
        for side in ("after", "before"):
            if s.get(side):
                kind, weight_, bias_ = s[side]
                s[side] = eden.Norm(weight_, bias_, kind, EPS)
        if op == "mx4_linear":
            s["weight"] = ctx.mx4_quantize(weight)
        elif op == "mx4_backward":
            s["weight_t"], s["x_t"] = ctx.mx4_quantize_transposed(weight), ctx.mx4_quantize_transposed(x)
    elif op == "mx4_linear":
        s["weight"] = _value4(weight)
    elif op == "mx4_backward":
        s["weight_t"], s["x_t"] = _value4(weight.t()), _value4(x.t())
    return s


# ------------------------------------------------------------------------------------ plain forms
def _grouped(v):
    rows, n = v.shape
    return torch.nn.functional.pad(v.float(), (0, -n % GROUP)).view(rows, _groups(n), GROUP)


def _code8(v):
    """8-bit form of v [rows, features] (int8 codes, uint8 exponents): the smallest 2^e with
    max|v| <= 127 * 2^e for each group."""
    rows, n = v.shape
    v = _grouped(v)
    e = ((v.abs().amax(dim=2).contiguous().view(torch.int32) + 0x1FFFF) >> 23) - 6
    e = e.clamp(min=1)
    codes = torch.round(v * ((254 - e) << 23).view(torch.float32)[:, :, None])
    return codes.to(torch.int8).view(rows, -1)[:, :n].contiguous(), e.to(torch.uint8)


def _value8(codes, exps):
    scale = (exps.to(torch.int32) << 23).view(torch.float32)
    return codes.float() * scale.repeat_interleave(GROUP, dim=1)[:, : codes.shape[1]]


def _value4(v):
    """What the 4-bit form of v [rows, features] stands for, in 32 bits."""
    rows, n = v.shape
    v = _grouped(v)
    # max = 1.f * 2^E needs 2^(E - 2), or 2^(E - 1) where 1.f is over 1.5
    e = (((v.abs().amax(dim=2).contiguous().view(torch.int32) + 0x3FFFFF) >> 23) - 2).clamp(min=1)
    u = v * ((254 - e) << 23).view(torch.float32)[:, :, None]
    size = u.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    u = torch.round(u / step) * step * (e << 23).view(torch.float32)[:, :, None]
    return u.view(rows, -1)[:, :n]


def _statistics(v, kind):
    """[rows, 2]: the mean (0 for rms) and one over the divisor."""
    mean = v.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    square = torch.square(v - mean).mean(dim=1, keepdim=True)
    return torch.cat([mean, 1 / torch.sqrt(square + EPS)], dim=1)


def _kept(m, n, drop, seed):
    """[m, n] truth values: Philox4x32-10 in 64-bit integers."""
    mask = 0xFFFFFFFF
    calls = _groups_of_8(n)
    c0 = torch.arange(calls, device="cuda").expand(m, calls)
    c1 = torch.arange(m, device="cuda")[:, None].expand(m, calls)
    c2, c3 = torch.full_like(c0, 3), torch.zeros_like(c0)
    k0, k1 = seed & mask, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & mask) ^ c1 ^ k0, b & mask, ((a >> 32) & mask) ^ c3 ^ k1, a & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    numbers = torch.stack([half for w in (c0, c1, c2, c3) for half in (w & 0xFFFF, w >> 16)], dim=2)
    return (numbers < int(65536 * (1 - drop) + 0.5)).view(m, -1)[:, :n]


def _groups_of_8(n):
    return -(-n // 8)


def _dropped(v, drop, seed):
    keep = int(65536 * (1 - drop) + 0.5)
    return torch.where(_kept(v.shape[0], v.shape[1], drop, seed), v * (65536 / keep), 0.0) if drop else v


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


def _normed(v, norm):
    kind, weight, bias = norm
    stats = _statistics(v, kind)
    y = (v - stats[:, :1]) * stats[:, 1:] * weight.float()
    return y if bias is None else y + bias.float(), stats


def _norm_backward(dy, v, stats, norm):
    """(gradient of v, of weight, of bias)"""
    kind, weight, bias = norm
    unit = (v - stats[:, :1]) * stats[:, 1:]
    g = dy * weight.float()
    inner = g - unit * (g * unit).mean(dim=1, keepdim=True)
    if kind == "layer":
        inner = inner - g.mean(dim=1, keepdim=True)
    return inner * stats[:, 1:], (dy * unit).sum(dim=0), dy.sum(dim=0) if bias is not None else None


def _run_plain(s):
    case, t, op = s["case"], s["type"], s["case"]["op"]
    if op == "join":
        u, after_stats = _normed(s["h"].float(), s["after"]) if s["after"] else (s["h"].float(), None)
        x = _dropped(u, case["drop"], s["seed"])
        if s["gate"] is not None:
            x = x * s["gate"].float()
        if s["residual"] is not None:
            x = x + s["scale"] * s["residual"].float()
        y, before_stats = _normed(x, s["before"]) if s["before"] else (None, None)
        out = {"x": x.to(t)}
        if y is not None:
            out["y"] = y.to(t)
        if case["train"]:
            out.update({name: v for name, v in (("after_stats", after_stats), ("before_stats", before_stats)) if v is not None})
        return out
    if op == "join_backward":
        held = lambda v: _value8(*v) if isinstance(v, tuple) else v.float()  # noqa: E731
        out, total = {}, s["dx"].float()
        if s["before"]:
            more, out["before_weight"], bias = _norm_backward(s["dy"].float(), held(s["x"]), s["before_stats"], s["before"])
            total = total + more
            if bias is not None:
                out["before_bias"] = bias
        if case["residual"]:
            out["residual"] = (s["scale"] * total).to(t)
        du = total
        if case["gate"] != "none":
            h = held(s["h"])
            if s["after"]:
                kind, weight, bias = s["after"]
                h = (h - s["after_stats"][:, :1]) * s["after_stats"][:, 1:] * weight.float()
                h = h if bias is None else h + bias.float()
            gate = total * _dropped(h, case["drop"], s["seed"])
            out["gate"] = gate.sum(dim=0) if case["gate"] == "vector" else gate.to(t)
            du = total * s["gate"].float()
        du = _dropped(du, case["drop"], s["seed"])
        if s["after"]:
            du, out["after_weight"], bias = _norm_backward(du, held(s["h"]), s["after_stats"], s["after"])
            if bias is not None:
                out["after_bias"] = bias
        out["h"] = du.to(t)
        return out
    if op == "dropout":
        y = _dropped(s["x"].float(), case["drop"], s["seed"])
        return {"y": (y if s["residual"] is None else y + s["residual"].float()).to(t)}
    if op == "mx4_quantize":
        return {"rows": _value4(s["x"]).to(t), "columns": _value4(s["x"].t()).to(t)}
    if op == "mx4_linear":
        y = _act(_value4(s["x"]) @ s["weight"].t() + s["bias"].float(), case["act"])
        return {"y": (y if s["residual"] is None else y + s["residual"].float()).to(t)}
    dx = _value4(s["dz"]) @ s["weight_t"].t()
    dx = dx * _act_slope(_value8(*s["pre"]), case["act"])
    return {"dx": dx.to(t), "bias_grad": dx.sum(dim=0), "weight_grad": _value4(s["dz"].t()) @ s["x_t"].t()}


def _run_own(s):
    case, ctx, t, op = s["case"], s["ctx"], s["type"], s["case"]["op"]
    if op == "join":
        j = ctx.block_join(s["h"], s["residual"], after=s["after"], before=s["before"], gate=s["gate"], scale=s["scale"], drop=case["drop"], seed=s["seed"],
                           out=s["out"][0], normed=s["out"][1], stats=case["train"])
        return {name: v for name, v in j._asdict().items() if v is not None}
    if op == "join_backward":
        d = ctx.block_join_backward(s["dx"], s["dy"], s["h"], s["x"], s["after_stats"], s["before_stats"], after=s["after"], before=s["before"], gate=s["gate"],
                                    scale=s["scale"], drop=case["drop"], seed=s["seed"], residual=None if case["residual"] else False)
        return {name: v for name, v in d._asdict().items() if v is not None}
    if op == "dropout":
        return {"y": ctx.dropout(s["x"], case["drop"], s["seed"], residual=s["residual"], out=s["out"])}
    if op == "mx4_quantize":
        rows, columns = ctx.mx4_quantize_both(s["x"])
        return {"rows": ctx.mx4_restore(rows, t), "columns": ctx.mx4_restore(columns, t)}
    if op == "mx4_linear":
        return {"y": ctx.mx4_linear(s["x"], s["weight"], s["bias"], act=case["act"], residual=s["residual"], out=s["out"])}
    dz, dz_t = ctx.mx4_quantize_both(s["dz"])
    dx, bias_grad = ctx.mx4_linear_input_grad(dz, s["weight_t"], pre=s["pre"], act=case["act"], out=s["out"], bias_grad=s["bias_grad"])
    return {"dx": dx, "bias_grad": bias_grad, "weight_grad": ctx.mx4_linear_weight_grad(dz_t, s["x_t"], out=s["weight_grad"])}


# ------------------------------------------------------------------------------------ 64 bits
def _exact_kept(m, n, drop, seed):
    """The keep factors, on the host in unsigned 64-bit arithmetic."""
    calls = (n + 7) // 8
    low = np.uint64(0xFFFFFFFF)
    word = [np.tile(np.arange(calls, dtype=np.uint64), m), np.repeat(np.arange(m, dtype=np.uint64), calls), np.full(m * calls, 3, np.uint64), np.zeros(m * calls, np.uint64)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        first, third = np.uint64(0xD2511F53) * word[0], np.uint64(0xCD9E8D57) * word[2]
        word = [(third >> np.uint64(32)) ^ word[1] ^ np.uint64(key[0]), third & low, (first >> np.uint64(32)) ^ word[3] ^ np.uint64(key[1]), first & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    numbers = np.stack([w.astype(np.uint32) for w in word], axis=1).view("<u2").reshape(m, calls * 8)[:, :n]
    below = round(65536 * (1 - drop))
    return torch.from_numpy(numbers < below).cuda().double() * (65536.0 / below)


def _exact_coded4(v):
    """What the 4-bit form of v [rows, cols] (64 bits) stands for: nearest of the eight magnitudes
    times the least power of two that holds the group, ties to the even place in the list."""
    n = v.shape[1]
    part = torch.cat([v, v.new_zeros(v.shape[0], -n % GROUP)], dim=1).unflatten(1, (-1, GROUP))
    mant, expo = torch.frexp(part.abs().amax(dim=2, keepdim=True) / 6)       # mant * 2^expo with 0.5 <= mant < 1
    expo = torch.where(mant == 0.5, expo - 1, expo).clamp(min=-126)
    unit = torch.ldexp(torch.ones_like(mant), expo)
    size = (part / unit).abs()
    sizes = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
    near = torch.zeros_like(size)
    for place in range(1, 8):
        middle = (sizes[place - 1] + sizes[place]) / 2
        reached = size >= middle if place % 2 == 0 else size > middle
        near = torch.where(reached, sizes[place], near)
    return (torch.copysign(near, part) * unit).flatten(1)[:, :n]


def _exact_held(v):
    if not isinstance(v, tuple):
        return v.double()
    codes, exps = v
    column = torch.arange(codes.shape[1], device=codes.device) // GROUP
    return torch.ldexp(codes.double(), exps[:, column].to(torch.int32) - 127)


def _exact_norm(v, kind):
    if kind == "layer":
        square, mean = torch.var_mean(v, dim=1, keepdim=True, correction=0)
    else:
        mean = v.new_zeros(v.shape[0], 1)
        square = torch.linalg.vecdot(v, v)[:, None] / v.shape[1]
    rate = torch.rsqrt(square + EPS)
    return (v - mean) * rate, torch.cat([mean, rate], dim=1)


def _exact_affine(unit, norm):
    return unit * norm[1].double() + (0.0 if norm[2] is None else norm[2].double())


def _exact_norm_gradient(g, unit, rate, kind):
    """rate * (g minus its projections on the unit row and, for layer norms, on the ones)"""
    n = g.shape[1]
    g = g - unit * (torch.linalg.vecdot(g, unit)[:, None] / n) - (g.sum(dim=1, keepdim=True) / n if kind == "layer" else 0.0)
    return g * rate


def _exact_act(z, act):
    return {
        "none": lambda: z,
        "relu": lambda: z.clamp(min=0),
        "gelu": lambda: z * 0.5 * torch.special.erfc(-z / 2 ** 0.5),
        "gelu_tanh": lambda: z * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)),
        "silu": lambda: z * torch.sigmoid(z),
    }[act]()


def _exact_slope(z, act):
    if act == "relu":
        return torch.heaviside(z, torch.zeros_like(z))
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad((_exact_act(z, act) * 1.0).sum(), z)[0]


def exact(case, seed):
    global own
    asked, own = own, False                                # the inputs, and the weights' values, without the framework
    try:
        s = prepare(case, seed)
    finally:
        own = asked
    m, n, op = case["m"], case["n"], case["op"]
    if op in ("join", "join_backward", "dropout"):
        kept = _exact_kept(m, n, case["drop"], s["seed"]) if case["drop"] else 1.0
    if op == "join":
        u, after_stats = s["h"].double(), None
        if s["after"]:
            u, after_stats = _exact_norm(u, case["after"])
            u = _exact_affine(u, s["after"])
        x = u * kept * (1.0 if s["gate"] is None else s["gate"].double())
        if case["residual"]:
            x = torch.add(x, s["residual"].double(), alpha=s["scale"])
        out = {"x": x}
        if s["before"]:
            unit, before_stats = _exact_norm(x, case["before"])
            out["y"] = _exact_affine(unit, s["before"])
        if case["train"] and s["after"]:
            out["after_stats"] = after_stats
        if case["train"] and s["before"]:
            out["before_stats"] = before_stats
        return out
    if op == "join_backward":
        out, total = {}, s["dx"].double()
        if s["before"]:
            dy, stats = s["dy"].double(), s["before_stats"].double()
            unit = (_exact_held(s["x"]) - stats[:, :1]) * stats[:, 1:]
            total = total + _exact_norm_gradient(dy * s["before"][1].double(), unit, stats[:, 1:], case["before"])
            out["before_weight"] = torch.einsum("mn,mn->n", dy, unit)
            if s["before"][2] is not None:
                out["before_bias"] = dy.sum(dim=0)
        if case["residual"]:
            out["residual"] = total * s["scale"]
        du = total * kept
        if s["h"] is not None:
            h = _exact_held(s["h"])
        if s["after"]:
            stats = s["after_stats"].double()
            unit = (h - stats[:, :1]) * stats[:, 1:]
            h = _exact_affine(unit, s["after"])
        if case["gate"] != "none":
            out["gate"] = du * h if case["gate"] == "matrix" else torch.einsum("mn,mn->n", du, h)
            du = du * s["gate"].double()
        if s["after"]:
            out["after_weight"] = torch.einsum("mn,mn->n", du, unit)
            if s["after"][2] is not None:
                out["after_bias"] = du.sum(dim=0)
            du = _exact_norm_gradient(du * s["after"][1].double(), unit, stats[:, 1:], case["after"])
        out["h"] = du
        return out
    if op == "dropout":
        return {"y": s["x"].double() * kept + (s["residual"].double() if case["residual"] else 0.0)}
    if op == "mx4_quantize":
        return {"rows": _exact_coded4(s["x"].double()), "columns": _exact_coded4(s["x"].double().t())}
    if op == "mx4_linear":
        weight = _exact_weights(case, seed)[0]
        y = _exact_act(torch.addmm(s["bias"].double(), _exact_coded4(s["x"].double()), _exact_coded4(weight).t()), case["act"])
        return {"y": y + (s["residual"].double() if case["residual"] else 0.0)}
    weight, x = _exact_weights(case, seed)
    dx = _exact_coded4(s["dz"].double()) @ _exact_coded4(weight.t().contiguous()).t()
    dx = dx * _exact_slope(_exact_held(s["pre"]), case["act"])
    return {"dx": dx, "bias_grad": dx.sum(dim=0), "weight_grad": _exact_coded4(s["dz"].double().t().contiguous()) @ _exact_coded4(x.t().contiguous()).t()}


def _exact_weights(case, seed):
    """The matrices that prepare quantises ahead of the call, drawn again in its order."""
    g, t = torch.Generator(device="cuda").manual_seed(seed), TYPES[case["dtype"]]
    m, n, k = case["m"], case["n"], case["k"]
    if case["op"] == "mx4_linear":
        _gauss(g, t, m, k)
        return _gauss(g, t, n, k, std=k ** -0.5).double(), None
    _laplace(g, t, m, n, std=0.02)
    return _gauss(g, t, n, k, std=k ** -0.5).double(), _gauss(g, t, m, k).double()
