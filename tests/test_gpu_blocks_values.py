"""Joins of rows whose values or sums lie at the ends of the range, and of what a mask leaves of them."""
import numpy as np
import pytest
import torch

from tests import blocks_reference as B
from tests import training_reference as R
from tests.test_gpu_training import normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.block_workspace_bytes(4096))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("n", [1024, 4096])
def test_rows_of_one_value_whose_sum_passes_the_range(ctx, n):
    """Such a row's mean is its value and its variance 0 (both exact here): what is left is the bias."""
    from paper_2108_08842_b200 import eden

    bias, weight = normal(1, n, dtype=torch.bfloat16), normal(2, n, dtype=torch.bfloat16)
    values = torch.tensor([1e36, -1e36, 3.3e38, 2.0 ** 120, 1.0, 0.0], dtype=torch.bfloat16, device="cuda")
    rows = values[:, None].repeat(1, n)
    for eps in (1e-6, 1e-12, 1.0):
        y, stats = ctx.norm(rows, eden.Norm(weight, bias, "layer", eps), stats=True)
        assert torch.equal(y, bias.expand_as(y))
        assert torch.equal(stats[:, 0], values.float())
        # the rate is one instruction's result, good to 2 units
        assert np.allclose(R.f64(stats[:, 1]), 1 / np.sqrt(np.float64(np.float32(eps))), rtol=2.0 ** -22, atol=0)


def test_rows_whose_squares_pass_the_range(ctx):
    """Far from each other, and next to one another: values around 1e36 are 2^112 apart."""
    from paper_2108_08842_b200 import eden

    n = 1024
    near = torch.full((n,), 1e36)
    near[::3] = 1.01e36
    rows = torch.stack([near, 1e36 * (-1.0) ** torch.arange(n), torch.cat([torch.tensor([3e38]), torch.zeros(n - 1)]), torch.randn(n, generator=torch.Generator().manual_seed(1)) * 1e37])
    rows = rows.to(torch.bfloat16).cuda()
    for kind in ("rms", "layer"):
        y, stats = ctx.norm(rows, eden.Norm(None, None, kind, 1e-6), stats=True)
        value, off, mean, rate, mean_off, rate_off = B.norm(R.f64(rows), np.zeros(rows.shape), kind, None, None, 1e-6)
        B.near(y, (value, off), R.UNIT[torch.bfloat16], R.TINY[torch.bfloat16])


# ------------------------------------------------------------------------------- masks
def all_dropped(m, n, drop, seed):
    gone = torch.from_numpy((B.kept(m, n, drop, seed) == 0).all(axis=1)).cuda()
    assert gone.any() and not gone.all()
    return gone


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("n", [1, 5, 8, 16])
def test_rows_of_which_the_mask_leaves_nothing(ctx, dtype, kind, n):
    """They are the residual's, whatever the block made; their gradients are 0, whatever came back."""
    from paper_2108_08842_b200 import eden

    m, drop, seed = 300, 0.9, 21
    gone = all_dropped(m, n, drop, seed)
    h, r, gate = normal(1, m, n, dtype=dtype), normal(2, m, n, dtype=dtype), normal(3, n, dtype=dtype)
    after, before = eden.Norm(normal(4, n, dtype=dtype), None, kind), eden.Norm(normal(5, n, dtype=dtype), None, kind)
    how = dict(after=after, before=before, gate=gate, drop=drop, seed=seed)
    clean = ctx.block_join(h, r, stats=True, **how)
    for bad in (float("nan"), float("inf")):
        broken = torch.where(gone[:, None], torch.full_like(h, bad), h)
        j = ctx.block_join(broken, r, stats=True, **how)
        assert torch.equal(j.x, clean.x) and torch.equal(j.y, clean.y) and torch.equal(j.before_stats, clean.before_stats)
    args = (h, clean.x, clean.after_stats, clean.before_stats)
    dx, dy = normal(6, m, n, dtype=dtype), normal(7, m, n, dtype=dtype)
    want = ctx.block_join_backward(dx, dy, *args, **how)
    assert (want.h[gone] == 0).all()
    for bad in (float("nan"), float("inf")):
        d = ctx.block_join_backward(dx, torch.where(gone[:, None], torch.full_like(dy, bad), dy), *args, **how)
        assert torch.equal(d.h, want.h) and torch.equal(d.after_weight, want.after_weight) and torch.equal(d.gate, want.gate)
