"""Joins on rows that end inside a chunk of 16 bytes, and results over the matrices that they come from."""
import pytest
import torch

from tests.test_gpu_blocks import Case, make
from tests.test_gpu_training import normal, within
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


def copies(c, *tensors):
    return [within(t.clone(), c.extra, 0) for t in tensors]


@pytest.mark.parametrize("drop", [0.0, 0.3])
@pytest.mark.parametrize("n,extra", [(1024, 0), (1001, 0), (264, 8), (40, 1)])
def test_gradients_in_place_without_norms(ctx, n, extra, drop):
    """Every result over every input that has a value for each of its own, one and all at a time."""
    c = Case(37, n, torch.bfloat16, "none", "none", "matrix", drop=drop, extra=extra)
    dx = make(5, 37, n, torch.bfloat16, extra)
    how = {k: v for k, v in c.how().items() if k != "gate"}
    want = ctx.block_join_backward(dx, None, c.h, gate=c.gate, **how)
    names = ("residual", "out", "gate_grad")
    for places in [(i, None, None) for i in range(3)] + [(None, i, None) for i in range(3)] + [(None, None, i) for i in range(3)] + [
            (0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0)]:
        held = copies(c, dx, c.h, c.gate)
        outs = {name: held[at] for name, at in zip(names, places) if at is not None}
        got = ctx.block_join_backward(held[0], None, held[1], gate=held[2], **outs, **how)
        assert all(torch.equal(getattr(got, f), getattr(want, f)) for f in ("residual", "h", "gate")), places


@pytest.mark.parametrize("n,extra", [(1024, 0), (1001, 0), (264, 8)])
def test_joins_in_place_without_norms(ctx, n, extra):
    c = Case(37, n, torch.float16, "none", "none", "matrix", drop=0.3, extra=extra)
    how = {k: v for k, v in c.how().items() if k != "gate"}
    want = ctx.block_join(c.h, c.residual, gate=c.gate, **how).x
    for place in range(3):
        held = copies(c, c.h, c.residual, c.gate)
        assert torch.equal(ctx.block_join(held[0], held[1], gate=held[2], out=held[place], **how).x, want)
    # one row: a vector gate has a value for each result too
    one, gate = make(3, 1, n, torch.float16), normal(4, n, dtype=torch.float16)
    want = ctx.block_join(one, gate=gate, drop=0.3, seed=1).x
    assert torch.equal(ctx.block_join(one, gate=gate, drop=0.3, seed=1, out=gate[None]).x, want)
