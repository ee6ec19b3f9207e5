"""A client's blocks with products in 4 bits: the weights, and the order of a step's calls."""
import numpy as np
import pytest
import torch

from tests import mx4_reference as M
from tests import training_reference as R
from tests.test_gpu_client_blocks import build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_weights_are_rounded_once(dtype):
    """The 4-bit weights are those of the fp32 parameters, by rows and by columns, also where these lie next
    to the middle between two codes and 16 bits would not tell on which side."""
    ctx, net, _, _ = build(16, 72, 100, 2, dtype=dtype, norm="rms", products="mx4")
    vector = net.vector.clone()
    matrices = [p for p in net.parts(vector) if p.dim() == 2]
    for p in matrices:
        p[:, 0], p[0] = 6.0, 6.0
        p[1:, 1:] = torch.where(p[1:, 1:] > 0, 2.5 * (1 + 2.0 ** -14), 0.75 * (1 - 2.0 ** -14))
    net.load(vector)
    for p, (rows, columns) in zip(matrices, net._mx4):
        for q, v in ((rows, R.f64(p)), (columns, R.f64(p).T)):
            codes, exps = M.unpack(q)
            want = M.quantise(v)
            assert np.array_equal(codes, want[0]) and np.array_equal(exps, want[1])
    ctx.close()


@pytest.mark.parametrize("norm,gate", [("rms", True), ("layer", False)])
def test_two_blocks_step_by_step(norm, gate):
    """Forward and backward of two blocks, every call with operands that this test makes of the parameters."""
    from paper_2108_08842_b200 import eden

    tokens, width, hidden, seed, drop = 130, 96, 200, 7, 0.2
    ctx, net, x, dy = build(tokens, width, hidden, 2, norm=norm, drop=drop, gate=gate, products="mx4")
    out, gradient = net.forward(x, seed=seed), net.backward(dy)
    at, parts = 0, {}

    def take(name, *shape):
        nonlocal at
        size = int(np.prod(shape))
        parts[name] = net.vector[at:at + size].view(shape)
        at += size

    for b in range(2):
        for name, shape in (("w1", (hidden, width)), ("b1", (hidden,)), ("w2", (width, hidden)), ("b2", (width,))):
            take((name, b), *shape)
    for b in range(2):
        for name in ("before", "after") + (("before bias", "after bias") if norm == "layer" else ()) + (("gate",) if gate else ()):
            take((name, b), width)
    assert at == net.d

    half = lambda name, b: parts[name, b].bfloat16() if (name, b) in parts else None  # noqa: E731
    norm_of = lambda side, b: eden.Norm(half(side, b), half(side + " bias", b), norm) if b < 2 else None  # noqa: E731
    rows = lambda name, b: ctx.mx4_quantize(parts[name, b])  # noqa: E731
    columns = lambda name, b: ctx.mx4_quantize_transposed(parts[name, b])  # noqa: E731
    joins = [dict(after=norm_of("after", b), before=norm_of("before", b + 1), gate=half("gate", b), drop=drop, seed=2 * seed + b) for b in range(2)]
    z = x
    y, first = ctx.norm(x, norm_of("before", 0), stats=True)
    kept = []
    for b in range(2):
        a, pre = ctx.mx4_linear(y, rows("w1", b), half("b1", b), act="gelu", save="pre")
        h = ctx.mx4_linear(a, rows("w2", b), half("b2", b))
        j = ctx.block_join(h, z, stats=True, **joins[b])
        kept.append((y, a, pre, h, j))
        z, y = j.x, j.y
    assert torch.equal(z, out)
    want, dx, dn = {}, dy, None
    for b in (1, 0):
        y, a, pre, h, j = kept[b]
        d = ctx.block_join_backward(dx, dn, ctx.checkpoint_save(h), None if b else ctx.checkpoint_save(j.x), j.after_stats, j.before_stats, **joins[b])
        want["after", b], want["after bias", b], want["gate", b] = d.after_weight, d.after_bias, d.gate
        if not b:
            want["before", 1], want["before bias", 1] = d.before_weight, d.before_bias
        want["b2", b] = ctx.act_backward(d.h, None, out=False)
        want["w2", b] = ctx.mx4_linear_weight_grad(ctx.mx4_quantize_transposed(d.h), ctx.mx4_quantize_transposed(a))
        dz, want["b1", b] = ctx.mx4_linear_input_grad(d.h, columns("w2", b), pre=pre, act="gelu")
        want["w1", b] = ctx.mx4_linear_weight_grad(ctx.mx4_quantize_transposed(dz), ctx.mx4_quantize_transposed(y))
        dx, dn = d.residual, ctx.mx4_linear_input_grad(dz, columns("w1", b))
    _, want["before", 0], want["before bias", 0] = ctx.norm_backward(dn, ctx.checkpoint_save(x), first, norm_of("before", 0), out=False)
    at = 0
    for key, part in parts.items():
        got = gradient[at:at + part.numel()].view(part.shape)
        at += part.numel()
        assert torch.equal(got, want[key][1] if isinstance(want[key], tuple) else want[key]), key
    assert ctx.status() == 0
    ctx.close()
