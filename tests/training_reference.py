"""The training operators in 64 bits on the CPU, from their definitions, and the error bounds
of the tests.

Bounds.  u(T) is half a unit in the last place of 1 in the type (2^-8 bf16, 2^-11 fp16, 2^-24
fp32).  A sum of n products held in fp32 is off by at most (n + 8) * 2^-23 * sum |a b| (twice
the classic n * 2^-24, since matrix units may cut instead of round).  Slopes and activations
are a handful of fp32 operations of at most 16 units each on quantities below 2, so they are
off by at most ACT = 2^-18, and activations by ACT * (1 + |z|).  All slopes are below 1.13.
"""
import math

import numpy as np
import torch

GROUP = 32
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
ACT = 2.0 ** -18
LIPSCHITZ = 1.13
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def f64(t):
    return t.detach().double().cpu().numpy()


_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, name):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "gelu":
        return z * 0.5 * (1 + _erf(z / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + np.exp(-z))
    return z.copy()


def slope(z, name):
    if name == "relu":
        return np.where(z > 0, 1.0, np.where(z <= 0, 0.0, z))
    if name == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        p = 1 / (1 + np.exp(-z))
        return p * (1 + z * (1 - p))
    return np.ones_like(z)


def code(v):
    """(int codes, exponent bytes) of a float64 matrix, group by group from the definition."""
    m, n = v.shape
    groups = -(-n // GROUP)
    codes, exps = np.zeros((m, n), np.int64), np.zeros((m, groups), np.int64)
    for g in range(groups):
        part = v[:, g * GROUP:(g + 1) * GROUP]
        bad = ~np.isfinite(part).all(axis=1)
        top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(part), part, 0.0)).max(axis=1))
        e = np.full(m, -126)
        for r in range(m):
            while top[r] > 127 * 2.0 ** float(e[r]):
                e[r] += 1
        exps[:, g] = np.where(bad, 255, e + 127)
        with np.errstate(invalid="ignore"):
            codes[:, g * GROUP:(g + 1) * GROUP] = np.where(bad[:, None], 0, np.rint(np.where(bad[:, None], 0.0, part) / 2.0 ** e[:, None].astype(float)))
    return codes, exps


def value(codes, exps):
    codes, exps = np.asarray(codes, np.float64), np.asarray(exps)
    e = exps[:, np.arange(codes.shape[1]) // GROUP]
    return np.where(e == 255, np.nan, codes * 2.0 ** (e - 127.0))


def restored(codes, exps, dtype):
    """What a checkpoint is restored to in a type: its values, saturated at the type's largest."""
    top = torch.finfo(dtype).max
    return np.clip(value(codes, exps), -top, top)


def held(saved):
    return value(saved[0].cpu().numpy(), saved[1].cpu().numpy().astype(np.int64))


def rounding(ref, dtype):
    """The largest error of rounding once to dtype."""
    return UNIT[dtype] * np.abs(ref) * (1 + 2.0 ** -7) + TINY[dtype]


def sum_bound(a, b):
    """Bound of the fp32 sums in a @ b."""
    return (a.shape[1] + 8) * 2.0 ** -23 * (np.abs(a) @ np.abs(b))


def near(got, ref, bound):
    got = f64(got)
    assert got.shape == ref.shape
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(got), nan)
    over = np.abs(got - ref)[~nan] - np.broadcast_to(bound, ref.shape)[~nan]
    assert over.size == 0 or over.max() <= 0, "%g over the bound" % over.max()
