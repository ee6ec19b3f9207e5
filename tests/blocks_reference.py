"""What joins a client's blocks, in 64 bits on the CPU from the definitions, each with a bound of the
kernels' error.

Bounds.  U = 2^-24 is half a unit of fp32.  A sum over a row or a column passes every term through at
most DEPTH additions behind a product (16 in a thread, 9 across a warp and its team, 7 across a
cluster), so it is off by at most DEPTH * U * sum |terms|; sums over m rows through m + DEPTH.  Errors
of the terms themselves are carried along to first order, with a factor of 2 on what a few fp32
operations add.
"""
import numpy as np
import torch

U = 2.0 ** -24
DEPTH = 48


def f64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------- dropout
def numbers(m, n, seed, first_row=0):
    """The 16-bit number of every value: Philox4x32-10."""
    calls = (n + 7) // 8
    c = [np.tile(np.arange(calls, dtype=np.uint64), m), np.repeat(np.arange(first_row, first_row + m, dtype=np.uint64), calls),
         np.full(m * calls, 3, np.uint64), np.zeros(m * calls, np.uint64)]
    k = [seed % 2 ** 32, seed // 2 ** 32]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack([w.astype(np.uint32) for w in c], axis=1).view("<u2").reshape(m, calls * 8)[:, :n]


def kept(m, n, drop, seed, first_row=0):
    """0, or 65536 over the number of numbers that keep a value."""
    below = int(65536 * (1 - drop) + 0.5)
    if below == 65536:
        return np.ones((m, n))
    return np.where(numbers(m, n, seed, first_row) < below, 65536.0 / max(below, 1), 0.0)


# ------------------------------------------------------------------------------- norms
def statistics(v, kind, eps):
    mean = v.mean(axis=1, keepdims=True) if kind == "layer" else np.zeros((len(v), 1))
    return mean, 1 / np.sqrt(np.square(v - mean).mean(axis=1, keepdims=True) + eps)


def norm(v, off, kind, weight, bias, eps):
    """(values, bound, mean, rate, bounds of both); off: the bound of v's own error."""
    mean, rate = statistics(v, kind, eps)
    mean_off = DEPTH * U * np.abs(v).mean(axis=1, keepdims=True) + off.mean(axis=1, keepdims=True) if kind == "layer" else 0 * mean
    inner = np.abs(v - mean)
    square_off = (2 * DEPTH * U * np.square(inner) + 2 * inner * (off + mean_off) + np.square(off + mean_off)).mean(axis=1, keepdims=True)
    rate_off = 0.5 * rate ** 3 * square_off + 8 * U * rate
    unit_off = rate * (off + mean_off + 4 * U * (np.abs(v) + np.abs(mean))) + inner * rate_off
    w, b = (1.0 if weight is None else weight), (0.0 if bias is None else bias)
    value = (v - mean) * rate * w + b
    return value, np.abs(w) * unit_off + 8 * U * (np.abs(inner * rate * w) + np.abs(b)), mean, rate, mean_off, rate_off


def join(h, residual, after, before, gate, scale, factor):
    """after, before: (kind, weight, bias, eps) or None; factor: `kept`.  A dict of (value, bound)."""
    out = {}
    u, off = h, np.zeros_like(h)
    if after:
        u, off, mean, rate, mean_off, rate_off = norm(u, off, *after)
        out["after_stats"] = np.concatenate([mean, rate], axis=1), np.concatenate([mean_off, rate_off], axis=1)
    g = 1.0 if gate is None else gate
    r = 0.0 if residual is None else scale * residual
    with np.errstate(invalid="ignore"):
        x = np.where(factor == 0, 0.0, u * factor) * g + r
        off = np.where(factor == 0, 0.0, off * factor * np.abs(g) + 8 * U * np.abs(u * factor * g)) + 8 * U * np.abs(r)
    out["x"] = x, off
    if before:
        y, off, mean, rate, mean_off, rate_off = norm(x, off, *before)
        out["y"] = y, off
        out["before_stats"] = np.concatenate([mean, rate], axis=1), np.concatenate([mean_off, rate_off], axis=1)
    return out


def norm_backward(dy, dy_off, v, stats, kind, weight):
    """(gradient of v, bound), and (values, bound) of what the weight's and the bias's gradients sum."""
    mean, rate = stats[:, :1], stats[:, 1:]
    unit = (v - mean) * rate
    unit_off = 4 * U * (np.abs(v) + np.abs(mean)) * rate
    w = 1.0 if weight is None else weight
    g, g_off = dy * w, dy_off * np.abs(w) + 2 * U * np.abs(dy * w)
    row = lambda a: a.mean(axis=1, keepdims=True)  # noqa: E731
    inner, inner_off = row(g * unit), row(2 * DEPTH * U * np.abs(g * unit) + g_off * np.abs(unit) + np.abs(g) * unit_off)
    outer, outer_off = (row(g), row(2 * DEPTH * U * np.abs(g) + g_off)) if kind == "layer" else (0.0, 0.0)
    d = rate * (g - outer - unit * inner)
    off = rate * (g_off + outer_off + np.abs(unit) * inner_off + np.abs(inner) * unit_off + 8 * U * (np.abs(g) + np.abs(outer) + np.abs(unit * inner)))
    return (d, off), (dy * unit, dy_off * np.abs(unit) + np.abs(dy) * unit_off + 2 * U * np.abs(dy * unit)), (dy, dy_off)


def column_sum(v, off):
    return v.sum(axis=0), (len(v) + DEPTH) * U * np.abs(v).sum(axis=0) + off.sum(axis=0)


def join_backward(dx, dy, h, x, after_stats, before_stats, after, before, gate, scale, factor):
    """Gradients of `join` as a dict of (value, bound); gate a vector or a matrix."""
    out = {}
    t, off = dx, np.zeros_like(dx)
    if before:
        (d, d_off), weights, biases = norm_backward(dy, np.zeros_like(dy), x, before_stats, before[0], before[1])
        t, off = t + d, d_off + 4 * U * (np.abs(t) + np.abs(d))
        out["before_weight"], out["before_bias"] = column_sum(*weights), column_sum(*biases)
    out["residual"] = scale * t, abs(scale) * off + 2 * U * np.abs(scale * t)
    du, du_off = t * factor, off * factor + 4 * U * np.abs(t * factor)
    if gate is not None:
        u, u_off = h, np.zeros_like(h)
        if after:
            w, b = (1.0 if after[1] is None else after[1]), (0.0 if after[2] is None else after[2])
            unit = (h - after_stats[:, :1]) * after_stats[:, 1:]
            u = unit * w + b
            u_off = np.abs(w) * 4 * U * (np.abs(h) + np.abs(after_stats[:, :1])) * after_stats[:, 1:] + 4 * U * (np.abs(unit * w) + np.abs(b))
        part, part_off = u * du, np.abs(u) * du_off + u_off * np.abs(du) + 2 * U * np.abs(u * du)
        out["gate"] = column_sum(part, part_off) if gate.ndim == 1 else (part, part_off)
        du, du_off = du * gate, du_off * np.abs(gate) + 2 * U * np.abs(du * gate)
    if after:
        (du, du_off), weights, biases = norm_backward(du, du_off, h, after_stats, after[0], after[1])
        out["after_weight"], out["after_bias"] = column_sum(*weights), column_sum(*biases)
    out["h"] = du, du_off
    return out


def near(got, ref, unit=0.0, tiny=0.0):
    """got within the bound of (value, bound), and a rounding to a type of that unit."""
    value, off = ref
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == value.shape
    nan = np.isnan(value)
    assert np.array_equal(np.isnan(got), nan)
    over = np.abs(got - value)[~nan] - (1.01 * off + unit * (np.abs(value) + off) + tiny + 1e-37)[~nan]
    assert over.size == 0 or over.max() <= 0, "%g over the bound" % over.max()
