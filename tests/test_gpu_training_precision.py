"""Errors of the training operators that the bounds of single sums do not show: what is lost along
long sums."""

import numpy as np
import pytest
import torch

from tests import training_reference as R

pytestmark = pytest.mark.gpu

FORMS = ["LINEAR_AUTO", "LINEAR_PAIR", "LINEAR_SINGLE", "LINEAR_NARROW"]


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(512, 512, 16384) + eden.linear_workspace_bytes(512, 16384, 512))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


@pytest.fixture(params=FORMS)
def form(ctx, request):
    from paper_2108_08842_b200 import eden

    ctx.set_option(eden.OPT_LINEAR_FORM, getattr(eden, request.param))
    yield request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, eden.LINEAR_AUTO)


@pytest.fixture(params=[0, 1])
def splits(ctx, request):
    from paper_2108_08842_b200 import eden

    ctx.set_option(eden.OPT_LINEAR_SPLITS, request.param)
    yield request.param
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 0)


# ------------------------------------------------------------------------------- long sums
# The tensor cores cut their fp32 sums off after every product of 16 steps.  A sum of like signs
# that grows evenly over N products loses N / 4 units of its last place in the mean (half a unit of
# what it has reached), a unit being at most 2^-23 of it.  Codes and bias gradients are to come of at
# most 512 steps at a time, N = 32: 2^-20; the additions of the parts round by 2^-24 each.  (What is
# added is cut off as well; products with 1 have too few bits for that.)
CUT = 2.0 ** -20


@pytest.mark.parametrize("depth", [4096, 16384])
@pytest.mark.parametrize("save", ["pre", "out"])
def test_codes_of_long_sums(ctx, form, splits, depth, save):
    """Sums of positive products with their own size subtracted as the bias: the codes of what is
    left show 2^-19 of the sums."""
    m, n = 64, 96
    g = torch.Generator(device="cuda").manual_seed(depth)
    x = torch.ones((m, depth), dtype=torch.float16, device="cuda")
    w = torch.rand((n, depth), generator=g, device="cuda").add_(0.5).half()
    sums = R.f64(x) @ R.f64(w).T
    bias = torch.from_numpy(-sums[0]).half().cuda()
    z = sums + R.f64(bias)
    y, saved = ctx.linear(x, w, bias, save=save)
    bound = (CUT + depth / 512 * 2.0 ** -24) * sums
    step = 2.0 ** (saved[1].cpu().numpy().astype(float)[:, np.arange(n) // 32] - 127)
    if save == "out":                                    # the result's own rounding comes between
        bound = bound + R.rounding(np.abs(z) + bound, torch.float16)
    assert (np.abs(R.held(saved) - z) <= step / 2 + bound).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1024, 2048, 4096])
def test_bias_gradients_of_long_sums(ctx, form, dtype, n):
    """A long sum is as good as its parts of 512, each the bias gradient of a call of its own: between
    them lie the additions of the parts and twice those of the rows (256 rows: five within 32, then
    eight), 2^-24 each at most."""
    from paper_2108_08842_b200 import eden

    m, k = 256, 200
    g = torch.Generator(device="cuda").manual_seed(n)
    dz = torch.rand((m, n), generator=g, device="cuda").add_(0.5).to(dtype)
    w = torch.rand((n, k), generator=g, device="cuda").add_(0.5).to(dtype)
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 1)
    whole, part = torch.empty(k, device="cuda"), torch.empty(k, device="cuda")
    ctx.linear_input_grad(dz, w, bias_grad=whole)
    parts = np.zeros(k)
    for i in range(0, n, 512):
        ctx.linear_input_grad(dz[:, i:i + 512], w[i:i + 512], bias_grad=part)
        parts += R.f64(part)
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 0)
    assert (np.abs(R.f64(whole) - parts) <= (n / 512 - 1 + 2 * 13) * 2.0 ** -24 * parts).all()
