"""What a client with norms keeps between its passes."""
import pytest
import torch

from tests.test_gpu_client_blocks import build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("products", ["half", "mx4"])
@pytest.mark.parametrize("norm,blocks", [("rms", 1), ("layer", 3)])
def test_all_that_is_held(norm, blocks, products):
    tokens, width = 256, 100
    ctx, net, x, dy = build(tokens, width, 320, blocks, norm=norm, products=products)
    assert net.held_bytes(whole=True) == 0
    net.forward(x)
    # the input's checkpoint, and mean and rate of every row for each of the 2 * blocks norms
    assert net.held_bytes(whole=True) - net.held_bytes() == tokens * (width + 4) + 2 * blocks * 8 * tokens
    net.backward(dy)
    before = torch.cuda.memory_allocated()
    kept = net.held_bytes(whole=True)
    net.forward(x, train=False)
    torch.cuda.synchronize()
    # nothing of it stays: what is allocated comes in units of 512 bytes
    assert net.held_bytes(whole=True) == net.held_bytes() == 0 and before - torch.cuda.memory_allocated() >= kept
    ctx.close()


def test_blocks_without_norms_hold_their_input_with_the_first():
    ctx, net, x, _ = build(64, 96, 160, 2)
    net.forward(x)
    assert net.held_bytes(whole=True) == net.held_bytes() > 0
    ctx.close()
