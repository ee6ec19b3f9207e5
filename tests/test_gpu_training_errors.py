"""What training calls refuse, and what is left behind by a call that fails."""
import ctypes

import pytest
import torch

from tests.test_gpu_training import normal

pytestmark = pytest.mark.gpu


def test_an_error_is_reported_once():
    """A launch that the runtime refuses (into a capture that was cut off) leaves nothing that the
    next, good call would report."""
    from paper_2108_08842_b200 import eden

    runtime = ctypes.CDLL("libcudart.so.12")
    side = torch.cuda.Stream()
    stream = ctypes.c_void_p(side.cuda_stream)
    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(256, 256, 256), stream=side)
    x, w = normal(1, 200, 256, dtype=torch.bfloat16), normal(2, 256, 256, dtype=torch.bfloat16)
    out = torch.empty((200, 256), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        want = c.linear(x, w).clone()
        side.synchronize()
        assert runtime.cudaStreamBeginCapture(stream, 1) == 0
        assert runtime.cudaStreamSynchronize(stream) != 0      # not allowed there: ends the capture
        with pytest.raises(eden.EdenError):
            c.linear(x, w, out=out)
        graph = ctypes.c_void_p()
        assert runtime.cudaStreamEndCapture(stream, ctypes.byref(graph)) != 0
        runtime.cudaGetLastError()
        c.linear(x, w, out=out)
        c.checkpoint_save(x)
        side.synchronize()
    assert torch.equal(out, want) and c.status() == 0
    c.close()


@pytest.mark.parametrize("act", ["none", "silu"])
def test_a_pre_activation_is_looked_at_whatever_the_activation(act):
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(64, 64, 64))
    dy, w = normal(1, 8, 64, dtype=torch.bfloat16), normal(2, 64, 48, dtype=torch.bfloat16)
    good, other = c.checkpoint_save(normal(3, 8, 64)), c.checkpoint_save(normal(4, 8, 48))
    c.act_backward(dy, good, act=act)
    dx, db = c.linear_input_grad(dy, w, pre=other, act=act)
    assert dx.shape == (8, 48) and db.shape == (48,)
    for bad in ("pre", dy, (good[0],), (dy, dy), (good[0].cpu(), good[1].cpu()), (good[0], good[1][:, :1]), other, (good[0][:4], good[1][:4])):
        with pytest.raises(ValueError):
            c.act_backward(dy, bad, act=act)
    for bad in ("pre", dy, (other[0], dy), good, (other[0].cpu(), other[1].cpu())):
        with pytest.raises(ValueError):
            c.linear_input_grad(dy, w, pre=bad, act=act)
    c.close()


def test_no_autograd_graph_is_recorded():
    """Parameters are taken as they are: gradients come from the calls for them."""
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(64, 64, 64))
    x, w = normal(1, 8, 64, dtype=torch.bfloat16), torch.nn.Parameter(normal(2, 64, 64, dtype=torch.bfloat16))
    y, pre = c.linear(x, w, act="gelu", save="pre")
    dx, db = c.linear_input_grad(y, w, pre=pre, act="gelu")
    assert not any(t.requires_grad for t in (y, *pre, dx, db)) and w.grad is None
    assert torch.equal(y, c.linear(x, w.detach(), act="gelu"))
    c.close()
