"""Joins on rows that end inside a chunk of 16 bytes."""
import pytest
import torch

from tests.test_gpu_blocks import Case, make
from tests.test_gpu_training_guards import Guarded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.block_workspace_bytes(4096))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("after,before", [("none", "none"), ("rms", "rms"), ("layer", "none"), ("none", "layer")])
@pytest.mark.parametrize("n", [1, 7, 33, 257, 1001])
def test_rows_that_start_but_do_not_end_on_16_bytes(ctx, dtype, after, before, n):
    """All rows of all matrices start on 16 bytes and are not a multiple of 8 long: the columns behind them, and
    what lies behind the last row, stay as they were."""
    extra = -n % 8
    for m, gate, drop in ((1, "none", 0.4), (5, "matrix", 0.0), (9, "vector", 0.4)):
        c = Case(m, n, dtype, after, before, gate, drop=drop, extra=extra)
        x, y = Guarded(m, n, dtype, extra), Guarded(m, n, dtype, extra) if c.before else None
        want = ctx.block_join(c.h.contiguous(), c.residual.contiguous(), stats=True, **c.how())
        got = ctx.block_join(c.h, c.residual, out=x.view, normed=y.view if y else None, **c.how())
        assert torch.equal(got.x, want.x) and (y is None or torch.equal(got.y, want.y))
        x.check()
        if y:
            y.check()
        dx, dy = make(5, m, n, dtype, extra), make(6, m, n, dtype, extra) if c.before else None
        kept = make(7, m, n, dtype, extra)
        halves = {name: Guarded(m, n, dtype, extra) for name in ("residual", "out") + (("gate_grad",) if gate == "matrix" else ())}
        args = (dx, dy, c.h, kept, want.after_stats, want.before_stats)
        d = ctx.block_join_backward(*args, **{k: g.view for k, g in halves.items()}, **c.how())
        for guarded in halves.values():
            guarded.check()
        alone = ctx.block_join_backward(*[t if t is None else t.contiguous() for t in args], **c.how())
        assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(d, alone))


@pytest.mark.parametrize("m,n", [(1, 33), (7, 1001), (40, 9)])
def test_dropout_of_rows_that_start_but_do_not_end_on_16_bytes(ctx, m, n):
    extra = -n % 8
    x, r, out = make(1, m, n, torch.float16, extra), make(2, m, n, torch.float16, extra), Guarded(m, n, torch.float16, extra)
    for residual in (None, r):
        want = ctx.dropout(x.contiguous(), 0.3, 5, residual=None if residual is None else r.contiguous())
        assert torch.equal(ctx.dropout(x, 0.3, 5, residual=residual, out=out.view), want)
        out.check()
