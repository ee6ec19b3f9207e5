"""A client whose blocks have norms, a gate, dropout and products in 4 bits: joins, linear layers and
checkpoints as they are used together."""
import numpy as np
import pytest
import torch

from tests import blocks_reference as B
from tests import training_reference as R

pytestmark = pytest.mark.gpu


def build(tokens, width, hidden, blocks, **how):
    from paper_2108_08842_b200 import client, eden

    ctx = eden.Context(0, workspace_bytes_=client.FeedForward.workspace_bytes(tokens, width, hidden))
    net = client.FeedForward(ctx, width, hidden, blocks, **how)
    g = torch.Generator(device="cuda").manual_seed(5)
    vector = net.vector + 0.1 * torch.randn(net.d, generator=g, device="cuda") * (net.vector != 0)
    for p in net.parts(vector):
        if p.dim() == 1:
            p.add_(0.1 * torch.randn(p.shape, generator=g, device="cuda"))
    net.load(vector)
    x, dy = (torch.randn((tokens, width), generator=g, device="cuda").to(net.dtype) for _ in range(2))
    return ctx, net, x, dy


def reference(net, x, dy, seed):
    """(result, gradients of the parts) in 64 bits, from the 16-bit weights, without checkpoints or 4 bits."""
    parts = [torch.from_numpy(R.f64(p)).requires_grad_(True) for p in net.work]
    tokens, width = x.shape
    z = torch.from_numpy(R.f64(x))

    def norm(v, weight, bias):
        if net.norm == "layer":
            v = v - v.mean(dim=1, keepdim=True)
        v = v / torch.sqrt(v.square().mean(dim=1, keepdim=True) + 1e-6) * weight
        return v if bias is None else v + bias

    for b in range(net.blocks):
        w1, b1, w2, b2 = parts[4 * b: 4 * b + 4]
        before, after, gate = net._vectors(parts, b)
        a = torch.nn.functional.gelu(norm(z, *before) @ w1.T + b1)
        u = norm(a @ w2.T + b2, *after) * torch.from_numpy(B.kept(tokens, width, net.drop, (seed * net.blocks + b) % 2 ** 64))
        z = z + (u if gate is None else u * gate)
    (z * torch.from_numpy(R.f64(dy))).sum().backward()
    return z.detach().numpy(), [p.grad.numpy() for p in parts]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,width,hidden,blocks,norm,drop,gate", [(96, 64, 160, 2, "rms", 0.0, False), (33, 40, 72, 1, "layer", 0.3, True),
                                                                      (130, 101, 50, 3, "rms", 0.1, True), (64, 256, 300, 2, "layer", 0.0, True)])
def test_gradient_vector_of_blocks_with_norms(dtype, tokens, width, hidden, blocks, norm, drop, gate):
    ctx, net, x, dy = build(tokens, width, hidden, blocks, dtype=dtype, seed=3, norm=norm, drop=drop, gate=gate)
    y = net.forward(x, seed=11)
    rows = torch.full((3, net.d), 9.0, device="cuda")
    got = net.backward(dy, rows[1])
    assert got.data_ptr() == rows[1].data_ptr() and (rows[0] == 9).all() and (rows[2] == 9).all()
    z, grads = reference(net, x, dy, 11)
    # As for blocks without norms: a checkpoint is off by 1.8 % in the mean, and a gradient meets those of
    # its own block (operand, slope, the values behind both norms) and three for each block above it; the
    # 16-bit roundings on the way are eight a block, below 2^-8 each.
    bound = 0.018 * (3 * blocks + 1) + 8 * blocks * 2.0 ** -8
    for got_part, ref in zip(net.parts(got), grads):
        assert np.linalg.norm(R.f64(got_part) - ref) <= bound * np.linalg.norm(ref)
    assert np.linalg.norm(R.f64(y) - z) <= 8 * blocks * 2.0 ** -8 * np.linalg.norm(z)
    twice = net.backward(dy, rows[1], accumulate=True)
    assert np.allclose(R.f64(twice), 2 * R.f64(net.backward(dy)), rtol=1e-6, atol=1e-6)
    again = net.forward(x, seed=11)
    assert torch.equal(again, y)
    eager = net.forward(x, train=False)
    assert net.held_bytes() == 0 and (torch.equal(eager, y) == (drop == 0.0))
    assert ctx.status() == 0
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,width,hidden,norm,gate", [(128, 256, 512, "rms", True), (65, 100, 333, "layer", False)])
def test_gradient_vector_in_4_bits(dtype, tokens, width, hidden, norm, gate):
    ctx, net, x, dy = build(tokens, width, hidden, 1, dtype=dtype, seed=3, norm=norm, drop=0.2, gate=gate, products="mx4")
    y = net.forward(x, seed=11)
    got = net.backward(dy)
    z, grads = reference(net, x, dy, 11)
    # Normal values are off by 12 % in the mean in 4 bits.  A gradient meets at most its two operands, the
    # weights that dz came through, and the four operands of the forward products behind the values it
    # reads: sqrt(7) * 0.12 = 0.32 where they are independent, and half as much again.
    for got_part, ref in zip(net.parts(got), grads):
        assert np.linalg.norm(R.f64(got_part) - ref) <= 0.48 * np.linalg.norm(ref)
    assert np.linalg.norm(R.f64(y) - z) <= 0.48 * np.linalg.norm(z)
    assert torch.equal(net.forward(x, seed=11), y) and torch.equal(net.backward(dy), got)
    assert torch.isfinite(net.forward(x, train=False)).all() and ctx.status() == 0
    ctx.close()


def test_held_activations_in_4_bits():
    ctx, net, x, _ = build(256, 128, 512, 1, norm="rms", products="mx4")
    net.forward(x)
    checkpoints = 256 * (512 + 128)                               # the pre-activation and the block's result
    columns = (128 + 512) * 256 // 2                              # both products' inputs by columns
    tiles = (128 // 128 + 512 // 128) * 1024                      # and their exponents
    assert net.held_bytes() == checkpoints + checkpoints // 32 + columns + tiles
    ctx.close()


@pytest.mark.parametrize("how", [dict(norm="rms", gate=True, drop=0.1), dict(norm="layer", products="mx4")], ids=str)
def test_rounds_of_training_run(how):
    from paper_2108_08842_b200 import client

    losses = client.run(clients=2, rounds=3, bits=2.0, tokens=256, width=128, hidden=256, blocks=2, say=lambda *_: None, **how)
    assert len(losses) == 3 and all(np.isfinite(losses))
