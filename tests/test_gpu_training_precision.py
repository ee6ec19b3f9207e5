"""Errors of the training operators that the bounds of single sums do not show: what is lost along
long sums, and relative errors of activations where they are small."""
import math

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
# what it has reached), a unit being at most 2^-23 of it.  Codes and 32-bit results are to come of at
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m", [1024, 1536, 4096])
def test_weight_gradients_of_many_tokens(ctx, form, dtype, m):
    """As above: between the whole and its parts of 512 tokens lie the additions of the parts."""
    from paper_2108_08842_b200 import eden

    n, k = 96, 200
    g = torch.Generator(device="cuda").manual_seed(m)
    dz = torch.rand((m, n), generator=g, device="cuda").add_(0.5).to(dtype)
    x = torch.rand((m, k), generator=g, device="cuda").add_(0.5).to(dtype)
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 1)
    whole = R.f64(ctx.linear_weight_grad(dz, x))
    parts = sum(R.f64(ctx.linear_weight_grad(dz[i:i + 512], x[i:i + 512])) for i in range(0, m, 512))
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 0)
    assert (np.abs(whole - parts) <= (m / 512 - 1) * 2.0 ** -24 * parts).all()


# ------------------------------------------------------------------------------- small results
# 2^a from an `a` of two roundings is off by at most |a| * 2^-23, doubled here; what else is in an
# activation (a polynomial good to 8e-7, its ten roundings, 2^x and 1/x to a unit or two) stays below 2^-19.
def relative(z, act):
    a = {"none": 0.0 * z, "relu": 0.0 * z, "gelu": z * z / 2, "gelu_tanh": 2 * math.sqrt(2 / math.pi) * (np.abs(z) + 0.044715 * np.abs(z) ** 3),
         "silu": np.abs(z)}[act] * math.log2(math.e)
    return 2.0 ** -19 + a * 2.0 ** -22


def slope_terms(z, act):
    """Magnitudes of the terms that a slope is the sum of."""
    if act == "gelu":
        return np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in z.ravel()]).reshape(z.shape) + np.abs(z) * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act in ("silu", "gelu_tanh"):
        c = math.sqrt(2 / math.pi)
        u, du = (z, np.ones_like(z)) if act == "silu" else (2 * c * (z + 0.044715 * z ** 3), 2 * c * (1 + 3 * 0.044715 * z * z))
        p = 1 / (1 + np.exp(-u))
        return p + np.abs(z) * p * (1 / (1 + np.exp(u))) * du
    return np.abs(R.slope(z, act))


def true_slope(z, act):
    """The slope in 64 bits without the cancellations of 1 + erf and 1 + tanh."""
    if act == "gelu":
        return np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in z.ravel()]).reshape(z.shape) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act in ("silu", "gelu_tanh"):
        c = math.sqrt(2 / math.pi)
        u, du = (z, np.ones_like(z)) if act == "silu" else (2 * c * (z + 0.044715 * z ** 3), 2 * c * (1 + 3 * 0.044715 * z * z))
        return 1 / (1 + np.exp(-u)) * (1 + z * du / (1 + np.exp(u)))
    return R.slope(z, act)


def true_act(z, act):
    if act == "gelu":
        return z * np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in z.ravel()]).reshape(z.shape)
    if act == "gelu_tanh":
        return z / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return R.act(z, act)


@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("dtype,most", [(torch.float16, 5.0), (torch.bfloat16, 9.0)])
@pytest.mark.parametrize("m", [4, 160])
def test_small_activations(ctx, act, dtype, most, m):
    """Every value through weights that pick it out: errors relative to the result."""
    n = 256
    z = torch.linspace(-most, most, m * n, device="cuda").to(dtype).view(m, n)
    got = ctx.linear(z, torch.eye(n, dtype=dtype, device="cuda"), act=act)
    ref = true_act(R.f64(z), act)
    bound = relative(R.f64(z), act) * np.abs(ref)
    R.near(got, ref, bound + R.rounding(np.abs(ref) + bound, dtype))


@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("n", [254, 256])
def test_small_slopes(ctx, act, n):
    """One row at a time: the bias gradient is the slope before its rounding."""
    eye = torch.eye(n, dtype=torch.float16, device="cuda")
    dy = torch.full((1, n), 1024.0, dtype=torch.float16, device="cuda")
    for e in range(-9, -3):                              # |z| up to 127 / 16
        codes = torch.arange(-127, 129, device="cuda").clamp_(max=127).to(torch.int8)[None, :n].contiguous()
        pre = codes, torch.full((1, -(-n // 32)), e + 127, dtype=torch.uint8, device="cuda")
        z = R.held(pre)
        ref = 1024.0 * true_slope(z, act)
        bound = 1024.0 * relative(z, act) * slope_terms(z, act)
        _, db = ctx.act_backward(dy, pre, act=act)
        R.near(db[None], ref, bound)
        dx, db = ctx.linear_input_grad(dy, eye, pre=pre, act=act)
        R.near(db[None], ref, bound)
        R.near(dx, ref, bound + R.rounding(np.abs(ref) + bound, torch.float16))


@pytest.mark.parametrize("m,n,k", [(40, 72, 64), (100, 130, 96)])
def test_weight_gradient_of_a_checkpoint_past_the_range_of_fp16(ctx, m, n, k):
    """A checkpoint is restored to the type of dz: fp16 saturates at 65504 and rounds below 2^-24."""
    g = torch.Generator(device="cuda").manual_seed(m)
    codes = torch.randint(-127, 128, (m, k), generator=g, device="cuda").to(torch.int8)
    exps = torch.randint(127 - 30, 127 + 13, (m, -(-k // 32)), generator=g, device="cuda").to(torch.uint8)
    dz = (torch.randn((m, n), generator=g, device="cuda") * 0.02).half()
    held = R.restored(codes.cpu().numpy(), exps.cpu().numpy().astype(np.int64), torch.float16)
    assert np.abs(held).max() == 65504 and ((np.abs(held) < 2.0 ** -24) & (held != 0)).any()
    xs = torch.from_numpy(held).half().double().numpy()
    a = R.f64(dz).T
    R.near(ctx.linear_weight_grad(dz, (codes, exps)), a @ xs, R.sum_bound(a, xs))
    # bf16 holds every one of them
    wide = dz.bfloat16()
    xs = R.value(codes.cpu().numpy(), exps.cpu().numpy().astype(np.int64))
    a = R.f64(wide).T
    R.near(ctx.linear_weight_grad(wide, (codes, exps)), a @ xs, R.sum_bound(a, xs))
