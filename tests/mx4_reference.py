"""Microscaled 4-bit floating point in 64 bits on the CPU, from the definition."""
import numpy as np
import torch

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(v):
    """(codes [m, n] 0..15, exponent bytes [m, groups]) of a float64 matrix, group by group."""
    m, n = v.shape
    codes, exps = np.zeros((m, n), np.int64), np.zeros((m, -(-n // 32)), np.int64)
    for g in range(exps.shape[1]):
        part = v[:, 32 * g:32 * g + 32]
        bad = ~np.isfinite(part).all(axis=1)
        part = np.where(bad[:, None], 0.0, part)
        top = np.abs(part).max(axis=1)
        e = np.full(m, -126)
        while (top > 6 * 2.0 ** e.astype(float)).any():
            e = np.where(top > 6 * 2.0 ** e.astype(float), e + 1, e)
        size = np.abs(part) / 2.0 ** e.astype(float)[:, None]
        # the nearest magnitude; of two as near, the one in an even place
        off = np.abs(size[:, :, None] - SIZES)
        near = off <= off.min(axis=2, keepdims=True)
        place = np.where(near, np.where(np.arange(8) % 2 == 0, 2, 1), 0).argmax(axis=2)
        codes[:, 32 * g:32 * g + 32] = np.where(bad[:, None], 0, place + 8 * np.signbit(part))
        exps[:, g] = np.where(bad, 255, e + 127)
    return codes, exps


def values(codes, exps):
    e = exps[:, np.arange(codes.shape[1]) // 32]
    return np.where(e == 255, np.nan, np.where(codes & 8, -1, 1) * SIZES[codes & 7] * 2.0 ** (e - 127.0))


def unpack(q):
    """(codes, exponent bytes) of an Mx4, out of its bytes and tiles as the header gives them; checks that
    codes past the last value are 0 and no spare exponent is NaN."""
    packed, tiles, n = q.codes.cpu().numpy().astype(np.int64), q.exps.cpu().numpy().astype(np.int64), q.features
    m = len(packed)
    codes = np.stack([packed & 15, packed >> 4], axis=2).reshape(m, -1)
    assert codes.shape[1] == -(-n // 32) * 32 and (codes[:, n:] == 0).all()
    groups = -(-n // 32)
    r, g = np.arange(m)[:, None], np.arange(groups)[None, :]
    at = (r // 128 * (-(-n // 256)) + g // 8) * 1024 + g // 4 % 2 * 512 + r % 32 * 16 + r // 32 % 4 * 4 + g % 4
    flat = tiles.reshape(-1)
    exps = flat[at]
    spare = np.ones(flat.shape, bool)
    spare[at.reshape(-1)] = False
    assert (flat[spare] != 255).all()
    return codes[:, :n], exps


def pack(codes, exps, like):
    """An Mx4 of the bytes of another program."""
    from paper_2108_08842_b200 import eden

    m, n = codes.shape
    wide = np.zeros((m, -(-n // 32) * 32), np.int64)
    wide[:, :n] = codes
    r, g = np.arange(m)[:, None], np.arange(exps.shape[1])[None, :]
    tiles = np.full(like.exps.numel(), 127, np.int64)
    tiles[(r // 128 * (-(-n // 256)) + g // 8) * 1024 + g // 4 % 2 * 512 + r % 32 * 16 + r // 32 % 4 * 4 + g % 4] = exps
    return eden.Mx4(torch.from_numpy((wide[:, ::2] | wide[:, 1::2] << 4).astype(np.uint8)).cuda(),
                    torch.from_numpy(tiles.astype(np.uint8)).view(like.exps.shape).cuda(), n)


def held(q):
    return values(*unpack(q))
