"""The formulas of the joins' gradients against central differences, on the CPU in 64 bits, and the
generator behind dropout."""
import numpy as np
import pytest

from tests import blocks_reference as B
from tests.conftest import read_golden

CASES = [("rms", "rms", "vector", True), ("layer", "layer", "matrix", True), ("none", "rms", "vector", False), ("layer", "none", "none", True),
         ("none", "none", "matrix", True), ("rms", "layer", "none", False)]


@pytest.mark.parametrize("after,before,gate,drop", CASES)
def test_gradients_against_differences(after, before, gate, drop):
    rng = np.random.default_rng(len(after) * 7 + len(before) * 3 + len(gate))
    m, n, eps, scale = 5, 12, 1e-3, 0.7
    v = {"h": rng.normal(size=(m, n)), "residual": rng.normal(size=(m, n)), "after_weight": rng.normal(size=n), "after_bias": rng.normal(size=n),
         "before_weight": rng.normal(size=n), "before_bias": rng.normal(size=n),
         "gate": rng.normal(size=n) if gate == "vector" else rng.normal(size=(m, n))}
    factor = B.kept(m, n, 0.3, 99) if drop else np.ones((m, n))
    dx, dy = rng.normal(size=(m, n)), rng.normal(size=(m, n)) if before != "none" else None
    norms = lambda v: [None if kind == "none" else (kind, v[name + "_weight"], v[name + "_bias"], eps) for kind, name in ((after, "after"), (before, "before"))]  # noqa: E731

    def loss(v):
        a, b = norms(v)
        out = B.join(v["h"], v["residual"], a, b, None if gate == "none" else v["gate"], scale, factor)
        return (out["x"][0] * dx).sum() + ((out["y"][0] * dy).sum() if before != "none" else 0.0)

    a, b = norms(v)
    out = B.join(v["h"], v["residual"], a, b, None if gate == "none" else v["gate"], scale, factor)
    stats = [out[s][0] if s in out else None for s in ("after_stats", "before_stats")]
    got = B.join_backward(dx, dy, v["h"], out["x"][0], *stats, a, b, None if gate == "none" else v["gate"], scale, factor)
    for name, (value, _) in got.items():
        step = 1e-6
        for _ in range(4):
            way = rng.normal(size=v[name].shape)
            up, down = ({**v, name: v[name] + s * step * way} for s in (1, -1))
            assert abs((loss(up) - loss(down)) / (2 * step) - (value * way).sum()) <= 1e-6 * (1 + np.abs(value * way).sum())


def test_the_generator_is_philox():
    """The known answers that the sender's generator is held to, where the counters can be reached: row
    and column blocks, stream 3."""
    rows = read_golden("philox4x32_10_kat.txt")
    assert rows                                              # the file is there; the counters below are ours
    n = B.numbers(3, 20, 0x0123456789ABCDEF)
    assert n.shape == (3, 20) and n.dtype == np.uint16
    # one call by hand: Python's whole numbers
    c, k = [1, 2, 3, 0], [0x89ABCDEF, 0x01234567]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    assert [c[j // 2] >> 16 * (j % 2) & 0xFFFF for j in range(8)] == list(n[2, 8:16])


def test_kept_share_and_mean():
    """2^17 numbers: a share p is off by at most 6 standard deviations, 6 * sqrt(p (1 - p) / 2^17) <= 0.0083."""
    for drop in (0.1, 0.5, 0.9):
        f = B.kept(64, 2048, drop, 5)
        assert abs((f > 0).mean() - (1 - drop)) <= 0.0083
    assert (B.kept(4, 9, 1.0, 3) == 0).all() and (B.kept(4, 9, 0.0, 3) == 1).all()
