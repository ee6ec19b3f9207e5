"""Gradient calls whose caller wants one of the two results."""
import pytest
import torch

from tests.test_gpu_training import normal, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(1100, 1100, 1100))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,extra,offset", [(0, 64, 0, 0), (1, 1, 0, 0), (5, 33, 1, 1), (40, 96, 0, 0), (333, 1000, 0, 0), (700, 512, 32, 32), (700, 512, 3, 5)])
def test_act_backward(ctx, act, dtype, m, n, extra, offset):
    dy = within(normal(m, m, n, dtype=dtype), extra, offset)
    pre = ctx.checkpoint_save(normal(n, m, n)) if act != "none" else None
    dz, db = ctx.act_backward(dy, pre, act=act)
    none, alone = ctx.act_backward(dy, pre, act=act, out=False)
    assert none is None and torch.equal(alone, db)
    given = torch.full((n,), 0.5, device="cuda")
    assert ctx.act_backward(dy, pre, act=act, out=False, bias_grad=given)[1] is given and torch.equal(given, db)
    ctx.act_backward(dy, pre, act=act, out=False, bias_grad=given, accumulate=True)
    assert torch.equal(given, db + db)
    before = ctx.launch_count
    alone, none = ctx.act_backward(dy, pre, act=act, bias_grad=False)
    assert none is None and torch.equal(alone, dz) and ctx.launch_count == before + (m > 0)
    out = torch.empty_like(dz)
    assert ctx.act_backward(dy, pre, act=act, out=out, bias_grad=False)[0] is out and torch.equal(out, dz)
    for bad in (dict(out=False, bias_grad=False), dict(bias_grad=False, accumulate=True), dict(out=True), dict(bias_grad=True)):
        with pytest.raises(ValueError):
            ctx.act_backward(dy, pre, act=act, **bad)


@pytest.mark.parametrize("m", [0, 7, 300])
def test_input_grad_without_its_bias_gradient(ctx, m):
    dz, w = normal(1, m, 200, dtype=torch.bfloat16), normal(2, 200, 136, dtype=torch.bfloat16)
    pre = ctx.checkpoint_save(normal(3, m, 136))
    dx, _ = ctx.linear_input_grad(dz, w, pre=pre, act="silu")
    assert torch.equal(ctx.linear_input_grad(dz, w, pre=pre, act="silu", bias_grad=False), dx)
    for bad in (dict(bias_grad=False, accumulate=True), dict(bias_grad=True), dict(out=False)):
        with pytest.raises(ValueError):
            ctx.linear_input_grad(dz, w, pre=pre, act="silu", **bad)
