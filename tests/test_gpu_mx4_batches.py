"""4-bit products of more tiles than there are places for: a block, or a pair of blocks, takes several
tiles one after the other, so that the second sums in tensor memory, and the columns that they share with
the first ones, are used.  Their results are those of the same product in strips of a tile for each block,
bit for bit: every value is one sum in an order of its own."""
import pytest
import torch

from tests.test_gpu_mx4 import varied
from tests.test_gpu_training import normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.mx4_workspace_bytes(4100, 4100, 700))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


# 256 x 256 tiles for pairs, 128 x 128 and 128 x 64 for single blocks: at least three tiles each
FORMS = {"LINEAR_PAIR": (3900, 3900), "LINEAR_SINGLE": (3000, 2500), "LINEAR_NARROW": (2500, 1500)}


@pytest.fixture(params=list(FORMS))
def form(ctx, request):
    from paper_2108_08842_b200 import eden

    ctx.set_option(eden.OPT_LINEAR_FORM, getattr(eden, request.param))
    yield request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, eden.LINEAR_AUTO)


def strips(m):
    """Rows in strips of 256, which no block has a second tile of."""
    return [slice(i, min(i + 256, m)) for i in range(0, m, 256)]


# one step of the sum; two and a part; what takes longer than an epilogue
@pytest.mark.parametrize("k", [64, 600, 2500])
@pytest.mark.parametrize("act,residual,save", [("none", False, "none"), ("none", True, "none"), ("gelu", True, "pre"), ("silu", False, "out"), ("none", False, "pre")])
def test_forward_of_several_tiles(ctx, form, k, act, residual, save):
    m, n = FORMS[form]
    x, w = varied(1, m, k, torch.bfloat16), ctx.mx4_quantize(normal(2, n, k, std=k ** -0.5))
    b, r = normal(3, n, dtype=torch.bfloat16), normal(4, m, n, dtype=torch.bfloat16) if residual else None
    for _ in range(2):
        got = ctx.mx4_linear(ctx.mx4_quantize(x), w, b, act=act, residual=r, save=save)
        for s in strips(m):
            want = ctx.mx4_linear(ctx.mx4_quantize(x[s]), w, b, act=act, residual=None if r is None else r[s], save=save)
            if save == "none":
                assert torch.equal(got[s], want)
            else:
                assert torch.equal(got[0][s], want[0]) and torch.equal(got[1].codes[s], want[1].codes) and torch.equal(got[1].exps[s], want[1].exps)


@pytest.mark.parametrize("n", [64, 600, 2500])
@pytest.mark.parametrize("act,residual", [("none", False), ("gelu", True), ("relu", False)])
def test_input_grad_of_several_tiles(ctx, form, n, act, residual):
    m, k = FORMS[form]
    dz, w = varied(1, m, n, torch.bfloat16), ctx.mx4_quantize_transposed(normal(2, n, k, std=n ** -0.5))
    r = normal(3, m, k, dtype=torch.bfloat16) if residual else None
    z = ctx.checkpoint_save(normal(4, m, k))
    got, sums = ctx.mx4_linear_input_grad(ctx.mx4_quantize(dz), w, residual=r, pre=z, act=act)
    for s in strips(m):
        part = type(z)(z.codes[s], z.exps[s])
        want = ctx.mx4_linear_input_grad(ctx.mx4_quantize(dz[s]), w, residual=None if r is None else r[s], pre=part, act=act, bias_grad=False, dtype=torch.bfloat16)
        assert torch.equal(got[s], want)
    # the column sums are of the values before their rounding: half a step, 2^-8, of each off at most, and the sums' own
    # roundings in fp32, as many as there are rows at most
    values = got.double()
    bound = (2.0 ** -8 + (m + 40) * 2.0 ** -24) * values.abs().sum(dim=0)
    assert ((sums.double() - values.sum(dim=0)).abs() <= bound).all()
    again, twice = ctx.mx4_linear_input_grad(ctx.mx4_quantize(dz), w, residual=r, pre=z, act=act)
    assert torch.equal(again, got) and torch.equal(twice, sums)


# up to 2048 terms are one sum in tensor memory: one of them, two, three
@pytest.mark.parametrize("m", [64, 600, 2500, 4100])
def test_weight_grad_of_several_tiles(ctx, form, m):
    n, k = FORMS[form]
    dz, x = ctx.mx4_quantize_transposed(varied(1, m, n, torch.bfloat16)), ctx.mx4_quantize_transposed(varied(2, m, k, torch.bfloat16))
    got = ctx.mx4_linear_weight_grad(dz, x)
    first = got.clone()
    ctx.mx4_linear_weight_grad(dz, x, out=got, accumulate=True)
    assert torch.equal(got, first + first)
    for s in strips(n):
        if s.start % 128 == 0:
            part = type(dz)(dz.codes[s], dz.exps[s.start // 128:-(-s.stop // 128)], dz.features)
            assert torch.equal(ctx.mx4_linear_weight_grad(part, x), first[s])
