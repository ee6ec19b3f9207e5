"""Joins of rows whose values or sums lie at the ends of the range."""
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
