"""What joins a client's blocks (norms, gate, dropout, residual) against 64-bit forms."""
import numpy as np
import pytest
import torch

from tests import blocks_reference as B
from tests import training_reference as R
from tests.test_gpu_training import gen, normal, untouched, within
from tests.test_gpu_training_guards import Guarded

pytestmark = pytest.mark.gpu

HALVES = [torch.bfloat16, torch.float16]
WORKSPACE = 32768


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.block_workspace_bytes(WORKSPACE))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


def make(seed, m, n, dtype, extra=0, offset=0, mean=0.0, std=1.0):
    scale = torch.exp(0.5 * torch.randn(n, generator=gen(seed + 1), device="cuda"))
    return within((normal(seed, m, n) * scale * std + mean).to(dtype), extra, offset)


def norm_of(kind, seed, n, dtype, bias, eps=1e-5):
    from paper_2108_08842_b200 import eden

    if kind == "none":
        return None, None
    w, b = (1 + 0.2 * normal(seed, n)).to(dtype), (0.3 * normal(seed + 1, n)).to(dtype) if bias else None
    return eden.Norm(w, b, kind, eps), (kind, R.f64(w), None if b is None else R.f64(b), eps)


class Case:
    """Inputs of a join, and what they stand for in 64 bits."""

    def __init__(self, m, n, dtype, after="rms", before="rms", gate="vector", residual=True, drop=0.25, bias=False, extra=0, offset=0, seed=1, first_row=0):
        self.m, self.n, self.dtype, self.extra, self.seed, self.drop, self.first_row = m, n, dtype, extra, 0xABCDEF0123 * seed, drop, first_row
        self.h = make(seed, m, n, dtype, extra, offset, mean=0.5)
        self.residual = make(seed + 10, m, n, dtype, extra, offset) if residual else None
        self.gate = {"none": None, "vector": normal(seed + 20, n, dtype=dtype), "matrix": make(seed + 20, m, n, dtype, extra, offset)}[gate]
        self.after, self.after_ref = norm_of(after, seed + 30, n, dtype, bias)
        self.before, self.before_ref = norm_of(before, seed + 40, n, dtype, bias)
        self.scale = 0.75
        self.factor = B.kept(m, n, drop, self.seed, first_row)
        self.out = lambda: within(torch.zeros((m, n), dtype=dtype, device="cuda"), extra, offset)

    def how(self):
        return dict(after=self.after, before=self.before, gate=self.gate, scale=self.scale, drop=self.drop, seed=self.seed, first_row=self.first_row)

    def reference(self):
        f = lambda t: None if t is None else R.f64(t)  # noqa: E731
        return B.join(f(self.h), f(self.residual), self.after_ref, self.before_ref, f(self.gate), self.scale, self.factor)


def check_join(ctx, c):
    x, y = c.out(), c.out() if c.before else None
    j = ctx.block_join(c.h, c.residual, out=x, normed=y, stats=True, **c.how())
    ref = c.reference()
    assert j.x is x and j.y is y and untouched(x, c.extra) and (y is None or untouched(y, c.extra))
    for name, value in j._asdict().items():
        assert (value is None) == (name not in ref), name
        if value is not None:
            half = name in ("x", "y")
            B.near(value, ref[name], R.UNIT[c.dtype] if half else B.U, R.TINY[c.dtype] if half else 0.0)


SIZES = [(1, 1), (1, 8), (3, 31), (2, 256), (5, 257), (4, 1000), (7, 1001), (300, 64), (2, 4096), (3, 4104), (160, 520), (450, 272), (2, 8200), (151, 4100),
         (1, 16390), (2, 32768)]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,n", SIZES)
def test_join_sizes(ctx, dtype, m, n):
    check_join(ctx, Case(m, n, dtype))
    check_join(ctx, Case(m, n, dtype, after="layer", before="layer", gate="matrix", bias=True, drop=0.5, seed=3))


PARTS = [("none", "none", "none", False, 0.0), ("none", "none", "vector", True, 0.5), ("none", "none", "matrix", False, 0.9), ("rms", "none", "none", False, 0.0),
         ("none", "rms", "none", True, 0.1), ("none", "layer", "none", False, 0.0), ("layer", "rms", "none", True, 0.3), ("rms", "layer", "vector", False, 0.0),
         ("layer", "none", "matrix", True, 0.2), ("rms", "rms", "matrix", True, 1.0)]


@pytest.mark.parametrize("after,before,gate,residual,drop", PARTS)
@pytest.mark.parametrize("m,n,extra,offset", [(9, 520, 0, 0), (9, 520, 8, 8), (9, 520, 1, 1), (200, 333, 0, 0), (3, 8192, 2, 4), (4, 6001, 3, 5)])
def test_join_parts_and_layouts(ctx, after, before, gate, residual, drop, m, n, extra, offset):
    for dtype in HALVES:
        check_join(ctx, Case(m, n, dtype, after, before, gate, residual, drop, bias=n % 2 == 0, extra=extra, offset=offset))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("after,before,gate,residual,drop", PARTS + [("rms", "rms", "vector", True, 0.25), ("layer", "layer", "matrix", True, 0.1)])
@pytest.mark.parametrize("m,n,extra,offset,held", [(1, 40, 0, 0, False), (33, 520, 0, 0, True), (33, 520, 8, 8, False), (200, 333, 0, 0, True), (40, 1001, 3, 5, False),
                                                  (3, 8192, 0, 0, True), (4, 6001, 1, 1, True), (2, 16390, 0, 0, False), (450, 256, 0, 0, True)])
def test_join_backward(ctx, dtype, after, before, gate, residual, drop, m, n, extra, offset, held):
    c = Case(m, n, dtype, after, before, gate, residual, drop, bias=n % 2 == 0, extra=extra, offset=offset, seed=5)
    dx, dy = make(60, m, n, dtype, extra, offset, std=0.02), make(70, m, n, dtype, extra, offset, std=0.02) if c.before else None
    x = make(80, m, n, dtype, extra, offset)
    keep = (lambda t: ctx.checkpoint_save(t)) if held else (lambda t: t)
    h, x = keep(c.h), keep(x)
    value = lambda t: R.held(t) if held else R.f64(t)  # noqa: E731
    stats = [None if ref is None else torch.from_numpy(np.concatenate(B.statistics(value(t), ref[0], ref[3]), axis=1)).float().cuda()
             for t, ref in ((h, c.after_ref), (x, c.before_ref))]
    f = lambda t: None if t is None else R.f64(t)  # noqa: E731
    ref = B.join_backward(f(dx), f(dy), value(h), value(x), f(stats[0]), f(stats[1]), c.after_ref, c.before_ref, f(c.gate), c.scale, c.factor)
    outs = dict(residual=c.out(), out=c.out())
    if gate == "matrix":
        outs["gate_grad"] = c.out()
    got = ctx.block_join_backward(dx, dy, h, x, *stats, **outs, **c.how())
    assert got.residual is outs["residual"] and got.h is outs["out"] and all(untouched(t, extra) for t in outs.values())
    for name, g in got._asdict().items():
        wanted = name in ref and not (name.endswith("bias") and n % 2)
        assert (g is None) == (not wanted), name
        if wanted:
            half = g.dtype == dtype
            B.near(g, ref[name], R.UNIT[dtype] if half else B.U, R.TINY[dtype] if half else 0.0)
    again = ctx.block_join_backward(dx, dy, h, x, *stats, **c.how())
    assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(got, again))       # bit for bit, in fresh memory
    sums = {k: v for k, v in got._asdict().items() if v is not None and v.dtype == torch.float32}
    if sums:
        # into views of a gradient vector, added, and alone
        where = {("gate_grad" if k == "gate" else k + "_grad"): torch.full((3 * n + 1,), 0.5, device="cuda")[n + 1:2 * n + 1] for k in sums}
        ctx.block_join_backward(dx, dy, h, x, *stats, residual=False, out=False, accumulate=True, **where, **c.how())
        for k, v in sums.items():
            w = where["gate_grad" if k == "gate" else k + "_grad"]
            assert torch.equal(w, v + 0.5) and (w._base[:n + 1] == 0.5).all() and (w._base[2 * n + 1:] == 0.5).all()


@pytest.mark.parametrize("dtype", HALVES)
def test_norm_and_its_gradient_alone(ctx, dtype):
    from paper_2108_08842_b200 import eden

    for kind, m, n in (("rms", 5, 300), ("layer", 64, 1024), ("layer", 3, 33), ("rms", 1, 1)):
        x, dy = make(1, m, n, dtype), make(2, m, n, dtype)
        norm, ref = norm_of(kind, 3, n, dtype, True)
        y, stats = ctx.norm(x, norm, stats=True)
        assert torch.equal(y, ctx.norm(x, norm)) and torch.equal(y, ctx.block_join(x, before=norm, out=False).y)
        value, off = B.norm(R.f64(x), np.zeros((m, n)), *ref)[:2]
        B.near(y, (value, off), R.UNIT[dtype], R.TINY[dtype])
        (d, d_off), weights, biases = B.norm_backward(R.f64(dy), np.zeros((m, n)), R.f64(x), R.f64(stats), ref[0], ref[1])
        more = make(4, m, n, dtype)
        for extra in (None, more):
            dx, dw, db = ctx.norm_backward(dy, x, stats, norm, dx=extra)
            total = d + (0 if extra is None else R.f64(extra))
            B.near(dx, (total, d_off + 8 * B.U * (np.abs(total) + np.abs(d))), R.UNIT[dtype], R.TINY[dtype])
        B.near(dw, B.column_sum(*weights), B.U)
        B.near(db, B.column_sum(*biases), B.U)
        assert ctx.norm_backward(dy, x, stats, eden.Norm(None, None, kind), out=False, weight_grad=torch.empty(n, device="cuda"))[0] is None


# ------------------------------------------------------------------------------- values at the edges
@pytest.mark.parametrize("dtype", HALVES)
def test_rows_that_are_large_small_far_from_zero_or_all_the_same(ctx, dtype):
    """A mean of 250 times the deviation costs fp32's digits in a difference of squares, but not here: rows
    of 16-bit numbers near 256 have differences that are exact."""
    from paper_2108_08842_b200 import eden

    n = 1024
    top = 60000.0 if dtype == torch.float16 else 3e18
    rows = torch.stack([torch.zeros(n), torch.full((n,), 3.0), torch.full((n,), top), 256 + 2 * torch.arange(n).float() % 8,
                        torch.cat([torch.tensor([top]), torch.zeros(n - 1)]), 2.0 ** -14 * torch.ones(n), (-1.0) ** torch.arange(n) * top]).to(dtype).cuda()
    for kind in ("rms", "layer"):
        y, stats = ctx.norm(rows, eden.Norm(None, None, kind, 1e-6), stats=True)
        value, off, mean, rate, mean_off, rate_off = B.norm(R.f64(rows), np.zeros(rows.shape), kind, None, None, 1e-6)
        B.near(y, (value, off), R.UNIT[dtype], R.TINY[dtype])
        B.near(stats, (np.concatenate([mean, rate], axis=1), np.concatenate([mean_off, rate_off], axis=1)), B.U)


def test_infinities_and_nan_stay_in_their_rows_and_dropped_ones_are_gone(ctx):
    from paper_2108_08842_b200 import eden

    m, n = 6, 520
    h = make(1, m, n, torch.bfloat16).clone()
    clean = ctx.block_join(h, after=eden.Norm(), before=eden.Norm(), drop=0.5, seed=9)
    h[1, 7], h[4, 300] = float("nan"), float("inf")
    got = ctx.block_join(h, after=eden.Norm(), before=eden.Norm(), drop=0.5, seed=9)
    rows = torch.tensor([0, 2, 3, 5], device="cuda")
    assert torch.equal(got.x[rows], clean.x[rows]) and torch.equal(got.y[rows], clean.y[rows])
    # row 1: NaN wherever the mask keeps, 0 where it drops; row 4: inf / inf at one place, finite / inf elsewhere
    keep = torch.from_numpy(B.kept(m, n, 0.5, 9) > 0).cuda()
    assert torch.equal(torch.isnan(got.x[1]), keep[1]) and (got.x[1][~keep[1]] == 0).all()
    where = torch.zeros(n, dtype=torch.bool, device="cuda")
    where[300] = True
    assert torch.equal(torch.isnan(got.x[4]), where & keep[4])
    # without a norm a dropped value leaves nothing, whatever it was, nor does its gradient
    bad = torch.where(keep, 1.0, float("nan")).bfloat16()
    gate = normal(2, n, dtype=torch.bfloat16)
    assert torch.equal(ctx.dropout(bad, 0.5, 9), torch.where(keep, 2.0, 0.0).bfloat16())
    d = ctx.block_join_backward(torch.ones_like(bad), None, bad, gate=gate, drop=0.5, seed=9)
    assert torch.isfinite(d.gate).all() and torch.isfinite(d.h).all()


def test_no_rows(ctx):
    from paper_2108_08842_b200 import eden

    h, norm = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), eden.Norm(torch.ones(64, device="cuda").bfloat16())
    j = ctx.block_join(h, h, after=norm, before=norm, drop=0.1, stats=True)
    assert all(t.shape == s for t, s in zip(j, [(0, 64), (0, 64), (0, 2), (0, 2)]))
    g = torch.full((64,), 3.0, device="cuda")
    d = ctx.block_join_backward(h, h, h, h, j.after_stats, j.before_stats, after=norm, before=norm, after_weight_grad=g)
    assert d.h.shape == (0, 64) and (g == 0).all() and (d.before_weight == 0).all()
    g.fill_(3.0)
    ctx.norm_backward(h, h, j.before_stats, norm, weight_grad=g, bias_grad=False, accumulate=True)
    assert (g == 3).all()


@pytest.mark.parametrize("n", [1024, 1001])
def test_results_in_place(ctx, n):
    c = Case(40, n, torch.bfloat16, after="layer", before="rms", bias=True)
    want = ctx.block_join(c.h, c.residual, **c.how())
    h, r = c.h.clone(), c.residual.clone()
    got = ctx.block_join(h, r, out=r, normed=h, **c.how())
    assert torch.equal(got.x, want.x) and torch.equal(got.y, want.y) and got.x is r and got.y is h
    dx, dy = make(5, 40, n, torch.bfloat16), make(6, 40, n, torch.bfloat16)
    j = ctx.block_join(c.h, c.residual, stats=True, **c.how())
    args = (c.h, j.x, j.after_stats, j.before_stats)
    want = ctx.block_join_backward(dx, dy, *args, **c.how())
    a, b = dx.clone(), dy.clone()
    got = ctx.block_join_backward(a, b, *args, residual=a, out=b, **c.how())
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and got.residual is a and got.h is b


@pytest.mark.parametrize("extra,offset", [(0, 0), (1, 1), (2, 3), (8, 8)])
@pytest.mark.parametrize("after,before,gate", [("rms", "layer", "matrix"), ("none", "rms", "vector"), ("layer", "none", "none"), ("none", "none", "matrix")])
def test_calls_write_their_outputs_only(ctx, after, before, gate, extra, offset):
    for m, n in ((1, 1), (3, 33), (40, 257), (9, 520), (2, 8200)):
        c = Case(m, n, torch.bfloat16, after, before, gate, bias=True)
        x, y = Guarded(m, n, torch.bfloat16, extra, offset), Guarded(m, n, torch.bfloat16, extra, offset)
        want = ctx.block_join(c.h, c.residual, stats=True, **c.how())
        got = ctx.block_join(c.h, c.residual, out=x.view, normed=y.view if c.before else None, stats=True, **c.how())
        assert torch.equal(got.x, want.x) and (got.y is None or torch.equal(got.y, want.y))
        for guarded in (x, y):
            guarded.check()
        dx, dy = make(5, m, n, torch.bfloat16), make(6, m, n, torch.bfloat16) if c.before else None
        halves = {name: Guarded(m, n, torch.bfloat16, extra, offset) for name in ("residual", "out") + (("gate_grad",) if gate == "matrix" else ())}
        sums = {name: Guarded(1, n, torch.float32, 0, offset) for name, there in (("after_weight_grad", c.after), ("after_bias_grad", c.after),
                                                                                  ("before_weight_grad", c.before), ("before_bias_grad", c.before)) if there}
        args = (dx, dy, c.h, want.x, want.after_stats, want.before_stats)
        d = ctx.block_join_backward(*args, **{k: g.view for k, g in halves.items()}, **{k: g.view[0] for k, g in sums.items()}, **c.how())
        for guarded in (*halves.values(), *sums.values()):
            guarded.check()
        assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(d, ctx.block_join_backward(*args, **c.how())))


# ------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("m,n,extra,offset", [(1, 1, 0, 0), (5, 64, 0, 0), (130, 999, 1, 3), (3, 20000, 0, 0), (66, 264, 8, 8)])
def test_dropout_is_the_generator(ctx, m, n, extra, offset):
    x = within(torch.ones((m, n), dtype=torch.float16, device="cuda"), extra, offset)
    for drop, seed, first in ((0.5, 1, 0), (0.1, 2 ** 64 - 1, 7), (0.75, 0x123456789, 2 ** 31 - 1), (1.0, 3, 0), (0.0, 3, 0)):
        y = ctx.dropout(x, drop, seed, first_row=first)
        assert np.array_equal(R.f64(y), B.kept(m, n, drop, seed, first).astype(np.float16).astype(np.float64))
    # by rows, as one, and after another norm-free part: the same mask
    cut = torch.cat([ctx.dropout(x[i:i + 1], 0.5, 77, first_row=i) for i in range(m)])
    assert torch.equal(cut, ctx.dropout(x, 0.5, 77))


def test_the_mask_of_a_join_is_that_of_dropout(ctx):
    """Whatever the kernel: rows that a warp, a block or a cluster holds."""
    from paper_2108_08842_b200 import eden

    for m, n in ((3, 100), (700, 512), (5, 5000), (2, 20000)):
        ones = torch.ones((m, n), dtype=torch.bfloat16, device="cuda")
        j = ctx.block_join(ones, after=eden.Norm(eps=0.0), before=eden.Norm(), drop=0.5, seed=42)
        assert torch.equal(j.x, ctx.dropout(ones, 0.5, 42))


def test_a_seed_on_the_device_and_captured_calls(ctx):
    from paper_2108_08842_b200 import eden

    side = torch.cuda.Stream()
    c = eden.Context(0, workspace_bytes_=eden.block_workspace_bytes(1024), stream=side)
    k = Case(50, 1000, torch.bfloat16, after="rms", before="layer", bias=True)
    k.how_ = {**k.how(), "seed": torch.tensor([5], dtype=torch.int64, device="cuda")}
    dx, dy = make(5, 50, 1000, torch.bfloat16), make(6, 50, 1000, torch.bfloat16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        def step():
            j = c.block_join(k.h, k.residual, stats=True, **k.how_)
            d = c.block_join_backward(dx, dy, k.h, j.x, j.after_stats, j.before_stats, **k.how_)
            return [j.x, j.y, d.h, d.residual, d.gate, d.after_weight, d.before_bias]
        step()
        with torch.cuda.graph(graph, stream=side):
            held = step()
        for seed in (5, 2 ** 40 + 3, -1):
            k.how_["seed"].fill_(seed)
            graph.replay()
            side.synchronize()
            j = ctx.block_join(k.h, k.residual, stats=True, **{**k.how_, "seed": seed % 2 ** 64})
            d = ctx.block_join_backward(dx, dy, k.h, j.x, j.after_stats, j.before_stats, **{**k.how_, "seed": seed % 2 ** 64})
            torch.cuda.synchronize()
            for a, b in zip(held, [j.x, j.y, d.h, d.residual, d.gate, d.after_weight, d.before_bias]):
                assert torch.equal(a, b)
    del graph
    assert c.status() == 0
    c.close()


def test_two_contexts_at_once(ctx):
    """Each has its own stream and workspace."""
    from paper_2108_08842_b200 import eden

    k = [Case(600, 700 + 100 * i, torch.bfloat16, seed=i + 1) for i in range(2)]
    args = []
    for c in k:
        j = ctx.block_join(c.h, c.residual, stats=True, **c.how())
        args.append((j.x, j.y, c.h, j.x, j.after_stats, j.before_stats))
    want = [ctx.block_join_backward(*a, **c.how()) for a, c in zip(args, k)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in k]
    others = [eden.Context(0, workspace_bytes_=eden.block_workspace_bytes(1024), stream=s) for s in streams]
    got = [[o.block_join_backward(*a, **c.how()) for o, a, c in zip(others, args, k)] for _ in range(20)]
    torch.cuda.synchronize()
    for g in got:
        for a, b in zip(g, want):
            assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(a, b))
    for o in others:
        assert o.status() == 0
        o.close()


def test_a_long_matrix_passes_32_bit_offsets(ctx):
    """Rows whose first value lies past 2^31 elements."""
    m, n, stride = 5, 512, (1 << 29) + 64
    whole = torch.zeros(4 * stride + n, dtype=torch.bfloat16, device="cuda")
    h = whole.as_strided((m, n), (stride, 1))
    h.copy_(make(1, m, n, torch.bfloat16))
    from paper_2108_08842_b200 import eden

    norm = eden.Norm()
    want = ctx.block_join(h.contiguous(), h.contiguous(), after=norm, before=norm, drop=0.5, seed=3)
    got = ctx.block_join(h, h, after=norm, before=norm, drop=0.5, seed=3)
    assert torch.equal(got.x, want.x) and torch.equal(got.y, want.y)
    assert torch.equal(ctx.dropout(h, 0.5, 3), ctx.dropout(h.contiguous(), 0.5, 3))


def test_too_small_a_workspace_is_refused():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(1, 1, 1))
    k = Case(600, 4096, torch.bfloat16)
    j = c.block_join(k.h, k.residual, stats=True, **k.how())           # needs none
    with pytest.raises(eden.EdenError):
        c.block_join_backward(j.x, j.y, k.h, j.x, j.after_stats, j.before_stats, **k.how())
    c.close()
