"""The training operators together: a client's step into EDEN's sender."""
import numpy as np
import pytest
import torch

from tests import training_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,width,hidden,blocks,act", [(96, 64, 160, 2, "gelu"), (33, 40, 72, 1, "silu"), (257, 100, 50, 3, "gelu_tanh")])
def test_gradient_vector_of_a_client(dtype, tokens, width, hidden, blocks, act):
    from paper_2108_08842_b200 import client, eden

    ctx = eden.Context(0, workspace_bytes_=client.FeedForward.workspace_bytes(tokens, width, hidden))
    net = client.FeedForward(ctx, width, hidden, blocks, act=act, dtype=dtype, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((tokens, width), generator=g, device="cuda").to(dtype)
    dy = torch.randn((tokens, width), generator=g, device="cuda").to(dtype)
    y = net.forward(x)
    rows = torch.full((3, net.d), 9.0, device="cuda")
    got = net.backward(dy, rows[1])
    assert got.data_ptr() == rows[1].data_ptr() and (rows[0] == 9).all() and (rows[2] == 9).all()

    # the same model in 64 bits, from the 16-bit weights, without checkpoints
    parts = [torch.from_numpy(R.f64(p)).requires_grad_(True) for p in net.work]
    z = torch.from_numpy(R.f64(x))
    for b in range(blocks):
        w1, b1, w2, b2 = parts[4 * b: 4 * b + 4]
        u = z @ w1.T + b1
        if act == "gelu":
            a = 0.5 * u * (1 + torch.erf(u / 2 ** 0.5))
        elif act == "silu":
            a = u * torch.sigmoid(u)
        else:
            a = torch.nn.functional.gelu(u, approximate="tanh")
        z = z + a @ w2.T + b2
    (z * torch.from_numpy(R.f64(dy))).sum().backward()
    # Relative errors of the pieces, added: an 8-bit checkpoint is off by half a step at most, a
    # step being at most max / 63.5 of its group, and by step / sqrt(12) in the mean, with max below
    # 4 standard deviations: 4 / 63.5 / sqrt(12) = 1.8 %.  A gradient meets the checkpoints of its own
    # block (two: its operand and the slope) and one slope for each block above; the 16-bit
    # roundings on the way, two a block and direction, are below 2^-8 each.
    bound = 0.018 * (blocks + 1) + 4 * blocks * 2.0 ** -8
    for got_part, ref in zip(net.parts(got), parts):
        r = ref.grad.numpy()
        assert np.linalg.norm(R.f64(got_part) - r) <= bound * np.linalg.norm(r)
    assert np.linalg.norm(R.f64(y) - z.detach().numpy()) <= 4 * blocks * 2.0 ** -8 * np.linalg.norm(z.detach().numpy())

    twice = net.backward(dy, rows[1], accumulate=True)
    assert np.allclose(R.f64(twice), 2 * R.f64(net.backward(dy)), rtol=1e-6, atol=1e-6)
    assert torch.equal(net.forward(x, train=False), y) and net.held_bytes() == 0
    assert ctx.status() == 0
    ctx.close()


def test_held_activations_take_half_of_16_bits():
    from paper_2108_08842_b200 import client, eden

    ctx = eden.Context(0, workspace_bytes_=client.FeedForward.workspace_bytes(256, 128, 512))
    net = client.FeedForward(ctx, 128, 512, 2)
    net.forward(torch.randn((256, 128), device="cuda").bfloat16())
    values = 2 * 256 * (128 + 512 + 512)                          # input, pre-activation, hidden
    assert net.held_bytes() == values + values // 32
    ctx.close()


@pytest.mark.parametrize("bits", [1.0, 4.0])
def test_rounds_of_training_through_the_sender_lower_the_loss(bits):
    from paper_2108_08842_b200 import client

    losses = client.run(clients=3, rounds=8, bits=bits, tokens=512, width=256, hidden=512, blocks=2, say=lambda *_: None)
    assert all(np.isfinite(losses)) and losses[-1] < 0.8 * losses[0], losses
