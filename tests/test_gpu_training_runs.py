"""Input and weight gradients over sums long enough to be added up in parts, in every form of the
products, and tiles whose last wave goes to a second launch."""
import pytest
import torch

from tests.test_gpu_training import check_input_grad, check_weight_grad

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(4500, 4500, 1100))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


@pytest.fixture
def forced(ctx, request):
    from paper_2108_08842_b200 import eden

    form, splits = request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, getattr(eden, form))
    ctx.set_option(eden.OPT_LINEAR_SPLITS, splits)
    yield request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, eden.LINEAR_AUTO)
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 0)


FORMS = [("LINEAR_AUTO", 0)] + [(f, s) for f in ("LINEAR_PAIR", "LINEAR_SINGLE", "LINEAR_NARROW") for s in (1, 2)]


@pytest.mark.parametrize("forced", FORMS, indirect=True)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,k,extra,offset", [(333, 600, 270, 0, 0), (333, 1100, 129, 0, 0), (270, 2100, 333, 3, 5), (65, 4160, 301, 1, 1),
                                                (256, 4160, 256, 16, 16)])
def test_input_gradients_with_bias_gradients_over_long_sums(ctx, forced, dtype, m, n, k, extra, offset):
    check_input_grad(ctx, dtype, m, n, k, "gelu", True, extra, offset)
    check_input_grad(ctx, dtype, m, n, k, "none", False, extra, offset)


@pytest.mark.parametrize("forced", FORMS, indirect=True)
@pytest.mark.parametrize("held", [True, False])
@pytest.mark.parametrize("m,n,k", [(2500, 130, 200), (4400, 96, 260)])
def test_weight_gradients_with_many_tokens_in_a_part(ctx, forced, held, m, n, k):
    check_weight_grad(ctx, torch.bfloat16, m, n, k, held)


def test_input_gradient_with_its_last_wave_in_parts():
    """80 tiles of 256 x 256 on 74 pairs of SMs."""
    from paper_2108_08842_b200 import eden

    m, n, k = 1270, 4096, 4000
    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(m, n, k))
    c.set_option(eden.OPT_LINEAR_FORM, eden.LINEAR_PAIR)
    before = c.launch_count
    dz, w = torch.zeros((m, n), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    c.linear_input_grad(dz, w, bias_grad=torch.empty(k, device="cuda"))
    assert c.launch_count == before + 3                    # whole tiles, the rest in parts, column sums
    check_input_grad(c, torch.bfloat16, m, n, k, "silu", True)
    assert c.status() == 0
    c.close()
