"""4-bit products whose groups' powers of two lie at the ends of the range."""
import numpy as np
import pytest
import torch

from tests import mx4_reference as M
from tests import training_reference as R
from tests.test_gpu_training import gen, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.mx4_workspace_bytes(200, 300, 1024))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


def powers(seed, m, n, low, high):
    """Normal values, each group of 32 times a power of two from 2^low to 2^high."""
    e = torch.randint(low, high + 1, (m, -(-n // 32)), generator=gen(seed + 1), device="cuda").double()
    return normal(seed, m, n).double().clamp(-3, 3) * torch.pow(2.0, e).repeat_interleave(32, dim=1)[:, :n]


# The groups' products and both powers of two multiply exactly, so the results are off by their sums' roundings
# alone, wherever these fit fp32.
@pytest.mark.parametrize("m", [1, 2, 5, 8, 13, 130])
@pytest.mark.parametrize("x,w", [((123, 124), (-12, -8)), ((60, 124), (-120, -70)), ((-12, -8), (122, 123)), ((-120, -70), (60, 123)), ((-110, -60), (-20, 60)),
                                 ((-126, -120), (100, 123)), ((40, 60), (50, 55))], ids=str)
def test_products_at_the_ends_of_the_range(ctx, m, x, w):
    n, k = 70, 200
    a, b = powers(m, m, k, *x).to(torch.bfloat16), powers(7, n, k, *w).float()
    wq = ctx.mx4_quantize(b)
    xq = ctx.mx4_quantize(a)
    xs, ws = M.held(xq), M.held(wq).T
    ref = xs @ ws
    assert np.isfinite(ref).all() and np.abs(ref).max() < 3e38
    bound = R.sum_bound(xs, ws) + R.rounding(ref, torch.bfloat16) + 1e-37
    for operand in (a, xq):
        R.near(ctx.mx4_linear(operand, wq), ref, bound)


def test_one_large_group_against_small_weights(ctx):
    """d = 4 * 4 * 32 of the largest power of two that bf16 has, times a small one."""
    for m in (1, 8, 40):
        x, w = torch.full((m, 32), 2.0 ** 126, dtype=torch.bfloat16, device="cuda"), torch.full((33, 32), 2.0 ** -10, device="cuda")
        for a, b in ((x, w), (torch.full_like(x, 2.0 ** -10), torch.full_like(w, 2.0 ** 126))):
            wq = ctx.mx4_quantize(b)
            for operand in (a, ctx.mx4_quantize(a)):
                assert (ctx.mx4_linear(operand, wq).double() == 2.0 ** 121).all()


def test_results_past_the_range_and_nan_groups(ctx):
    """Infinity only where the result is; NaN groups stay NaN next to the largest powers of two."""
    for m in (1, 8):
        x, w = torch.full((m, 96), 1.0, dtype=torch.bfloat16, device="cuda"), torch.full((33, 96), 1.0, device="cuda")
        x[:, :32], w[:, :32] = 2.0 ** 126, 2.0 ** 10
        w[5, :32], w[9, 40] = 2.0 ** -126, float("nan")
        x[m - 1, 64:] = 2.0 ** -126
        w[7, 70] = float("inf")
        for operand in (x, ctx.mx4_quantize(x)):
            y = ctx.mx4_linear(operand, ctx.mx4_quantize(w))
            nan = torch.zeros((m, 33), dtype=torch.bool, device="cuda")
            nan[:, 9] = nan[:, 7] = True
            assert torch.equal(torch.isnan(y), nan)
            assert torch.isinf(y[:, [0, 1, 2, 3, 4, 6, 8, 10, 32]]).all() and torch.isfinite(y[:, 5]).all()
