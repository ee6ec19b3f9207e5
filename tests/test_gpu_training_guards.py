"""No training call writes outside its outputs: every output is a view into a buffer whose other
bytes are compared afterwards."""
import numpy as np
import pytest
import torch

from tests import training_reference as R
from tests.test_gpu_training import normal, within

pytestmark = pytest.mark.gpu

# rows of a remainder tile reach 255 rows past the end
GUARD_ROWS, GUARD = 256, 4096


class Guarded:
    """A matrix (or vector, m = 1) inside a buffer with a guard before and after it."""

    def __init__(self, m, n, dtype, extra=0, offset=0):
        self.m, self.n, self.row, self.at = m, n, n + extra, GUARD + offset
        size = self.at + (m + GUARD_ROWS) * self.row + GUARD
        self.whole = torch.randint(-128, 128, (size * torch.empty(0, dtype=dtype).element_size(),), dtype=torch.int8, device="cuda")
        self.buffer = self.whole.view(dtype)
        self.view = self.buffer[self.at:self.at + m * self.row].view(m, self.row)[:, :n]
        self.before = self.whole.clone()

    def check(self):
        """Everything but the view is as it was."""
        now = self.before.clone().view(self.buffer.dtype)
        now[self.at:self.at + self.m * self.row].view(self.m, self.row)[:, :self.n] = self.view
        assert torch.equal(now.view(torch.int8), self.whole)


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(1100, 1100, 1100))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


@pytest.fixture(params=[("LINEAR_AUTO", 0), ("LINEAR_FEW", 0), ("LINEAR_PAIR", 1), ("LINEAR_PAIR", 2), ("LINEAR_SINGLE", 1), ("LINEAR_SINGLE", 4),
                        ("LINEAR_NARROW", 1), ("LINEAR_NARROW", 8)], ids=lambda p: "%s-%d" % p)
def form(ctx, request):
    from paper_2108_08842_b200 import eden

    ctx.set_option(eden.OPT_LINEAR_FORM, getattr(eden, request.param[0]))
    ctx.set_option(eden.OPT_LINEAR_SPLITS, request.param[1])
    yield request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, eden.LINEAR_AUTO)
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 0)


LAYOUTS = [(0, 0), (1, 1), (3, 5), (8, 8), (32, 32)]
SIZES = [(1, 1, 1), (1, 96, 128), (3, 33, 1000), (13, 131, 1000), (32, 64, 520), (33, 257, 129), (130, 200, 264), (300, 520, 1000)]


@pytest.mark.parametrize("extra,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_linear(ctx, form, dtype, extra, offset):
    for m, n, k in SIZES:
        x, w, b, r = normal(m, m, k, dtype=dtype), normal(n, n, k, dtype=dtype, std=k ** -0.5), normal(k, n, dtype=dtype), normal(7, m, n, dtype=dtype)
        for save in ("none", "pre", "out"):
            out = Guarded(m, n, dtype, extra, offset)
            if save == "none":
                ctx.linear(x, w, b, act="silu", residual=r, out=out.view)
                out.check()
                continue
            codes, exps = Guarded(m, n, torch.int8, extra, offset), Guarded(m, -(-n // 32), torch.uint8, extra, offset)
            got, saved = ctx.linear(x, w, b, act="silu", residual=r, out=out.view, save=save, saved=(codes.view, exps.view))
            assert got is out.view and saved[0] is codes.view and saved[1] is exps.view
            for guarded in (out, codes, exps):
                guarded.check()
            fresh, kept = ctx.linear(x, w, b, act="silu", residual=r, save=save)
            # in fresh matrices: the same values
            assert torch.equal(fresh, got) and torch.equal(kept[0], codes.view) and torch.equal(kept[1], exps.view)


@pytest.mark.parametrize("extra,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients(ctx, form, dtype, extra, offset):
    for m, n, k in SIZES:
        dz, w, pre = normal(m, m, n, dtype=dtype, std=0.02), normal(n, n, k, dtype=dtype), ctx.checkpoint_save(normal(m + k, m, k))
        dx, db = Guarded(m, k, dtype, extra, offset), Guarded(1, k, torch.float32, 0, offset)
        ctx.linear_input_grad(dz, w, pre=pre, act="gelu", out=dx.view, bias_grad=db.view[0])
        dx.check()
        db.check()
        ctx.linear_input_grad(dz, w, pre=pre, act="gelu", out=dx.view, bias_grad=db.view[0], accumulate=True)
        db.check()
        dw = Guarded(n, k, torch.float32, extra, offset)
        for x in (pre, normal(k, m, k, dtype=dtype)):
            ctx.linear_weight_grad(dz, x, out=dw.view)
            dw.check()
            ctx.linear_weight_grad(dz, x, out=dw.view, accumulate=True)
            dw.check()


@pytest.mark.parametrize("extra,offset", LAYOUTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m,n", [(1, 1), (3, 33), (9, 1000), (257, 96), (40, 520)])
def test_checkpoints_and_activation_gradients(ctx, dtype, m, n, extra, offset):
    x = within(normal(m, m, n, dtype=dtype), extra, offset)
    codes, exps, back = Guarded(m, n, torch.int8, extra, offset), Guarded(m, -(-n // 32), torch.uint8, extra, offset), Guarded(m, n, dtype, extra, offset)
    saved = ctx.checkpoint_save(x, (codes.view, exps.view))
    ctx.checkpoint_restore(saved, dtype, back.view)
    for guarded in (codes, exps, back):
        guarded.check()
    want, scale = R.code(R.f64(x))
    assert np.array_equal(codes.view.cpu().numpy(), want) and np.array_equal(exps.view.cpu().numpy(), scale)
    if dtype == torch.float32:
        return
    for accumulate in (False, True):
        dz, db = Guarded(m, n, dtype, extra, offset), Guarded(1, n, torch.float32, 0, offset)
        db.view.fill_(0.5)
        ctx.act_backward(x, saved, act="silu", out=dz.view, bias_grad=db.view[0], accumulate=accumulate)
        dz.check()
        db.check()
