"""Microscaled 4-bit floating point: quantisation and products, against 64-bit forms.

Bounds of the products as in training_reference: the values and scales are multiplied exactly, and sums
of n products are off by at most (n + 8) * 2^-23 * sum |a b|.
"""
import numpy as np
import pytest
import torch

from tests import mx4_reference as M
from tests import training_reference as R
from tests.test_gpu_training import gen, normal, untouched, within
from tests.test_gpu_training_guards import Guarded

pytestmark = pytest.mark.gpu

HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.mx4_workspace_bytes(2100, 4200, 4200))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


@pytest.fixture(params=["LINEAR_AUTO", "LINEAR_PAIR", "LINEAR_SINGLE", "LINEAR_NARROW"])
def form(ctx, request):
    from paper_2108_08842_b200 import eden

    ctx.set_option(eden.OPT_LINEAR_FORM, getattr(eden, request.param))
    yield request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, eden.LINEAR_AUTO)


def varied(seed, m, n, dtype):
    """Groups of unequal size."""
    return (normal(seed, m, n) * torch.exp(2 * torch.randn((m, -(-n // 32)), generator=gen(seed + 7), device="cuda")).repeat_interleave(32, dim=1)[:, :n]).to(dtype)


# ------------------------------------------------------------------------------- quantisation
LAYOUTS = [(1, 1, 0, 0), (3, 31, 0, 0), (2, 32, 0, 0), (5, 33, 1, 1), (128, 256, 0, 0), (129, 257, 7, 3), (130, 96, 16, 16), (40, 1000, 0, 0), (300, 520, 32, 32),
           (257, 130, 3, 0), (1, 4128, 0, 0), (600, 1, 0, 0)]


@pytest.mark.parametrize("dtype", HALVES + [torch.float32])
@pytest.mark.parametrize("m,n,extra,offset", LAYOUTS)
def test_quantisation_is_the_definition(ctx, dtype, m, n, extra, offset):
    x = within(varied(n, m, n, dtype), extra, offset)
    rows, columns = ctx.mx4_quantize_both(x)
    for q, v in ((rows, R.f64(x)), (columns, R.f64(x).T)):
        codes, exps = M.unpack(q)
        want = M.quantise(v)
        assert np.array_equal(codes, want[0]) and np.array_equal(exps, want[1])
        out = within(torch.zeros(v.shape, dtype=dtype, device="cuda"), extra, offset)
        back = ctx.mx4_restore(q, dtype, out)
        assert back is out and untouched(out, extra)
        R.near(back, M.values(*want), R.TINY[dtype])                     # exact; below the smallest number rounded
    for alone, both in ((ctx.mx4_quantize(x), rows), (ctx.mx4_quantize_transposed(x), columns)):
        assert all(torch.equal(a, b) for a, b in zip(alone[:2], both[:2])) and alone.features == both.features


@pytest.mark.parametrize("dtype", HALVES + [torch.float32])
def test_quantisation_of_special_values(ctx, dtype):
    info = torch.finfo(dtype)
    rows = [[0.0] * 40, [-0.0] * 40, [info.max, -info.max, 1.0] + [0.0] * 37, [info.smallest_normal, -info.smallest_normal / 2] + [0.0] * 38,
            [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -5.0, 0.2, 4.99, 5.01] + [0.0] * 27, [6.25] + [1.0] * 39, [12.0, 0.5, 1.5, 7.0, 10.0] + [0.0] * 35,
            [float("inf")] + [1.0] * 39, [1.0] * 32 + [float("nan")] * 8, [1.0] * 39 + [float("-inf")], [1e-3] * 32 + [6.0] * 8]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype).cuda()
    for q, v in ((ctx.mx4_quantize(x), R.f64(x)), (ctx.mx4_quantize_transposed(x), R.f64(x).T)):
        codes, exps = M.unpack(q)
        want = M.quantise(v)
        assert np.array_equal(codes, want[0]) and np.array_equal(exps, want[1])
        R.near(ctx.mx4_restore(q, dtype), np.clip(M.values(*want), -float(info.max), float(info.max)), R.TINY[dtype])


def test_every_code_and_exponent_is_restored(ctx):
    codes = np.arange(256)[None, :].repeat(40, axis=0) % 16
    exps = (1 + np.arange(40 * 8).reshape(40, 8) % 255)
    q = M.pack(codes, exps, ctx.mx4_empty(40, 256))
    top = float(torch.finfo(torch.float32).max)
    R.near(ctx.mx4_restore(q, torch.float32), np.clip(M.values(codes, exps), -top, top), 0.0)


def test_quantisation_writes_its_outputs_only(ctx):
    from paper_2108_08842_b200 import eden

    for m, n in ((3, 33), (130, 300), (257, 1000)):
        x = normal(m, m, n, dtype=torch.bfloat16)
        guards = []
        for rows, features in ((m, n), (n, m)):
            codes = Guarded(rows, -(-features // 32) * 16, torch.uint8, 32, 16)
            exps = Guarded(1, -(-rows // 128) * -(-features // 256) * 1024, torch.uint8, 0, 16)
            guards.append((codes, exps, eden.Mx4(codes.view, exps.view.view(-(-rows // 128), -(-features // 256), 1024), features)))
        got = ctx.mx4_quantize_both(x, guards[0][2], guards[1][2])
        want = ctx.mx4_quantize_both(x)
        for g, w, (codes, exps, q) in zip(got, want, guards):
            assert g is q and torch.equal(q.codes, w.codes) and torch.equal(q.exps, w.exps)
            codes.check()
            exps.check()
        back = Guarded(m, n, torch.bfloat16, 3, 1)
        ctx.mx4_restore(got[0], torch.bfloat16, back.view)
        back.check()


# ------------------------------------------------------------------------------- forward
SIZES = [(1, 1, 1), (1, 64, 64), (3, 33, 1000), (8, 131, 520), (9, 70, 4100), (13, 131, 1000), (128, 128, 256), (130, 200, 264), (257, 300, 2049), (300, 520, 1000)]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear(ctx, form, dtype, m, n, k):
    x, w = within(varied(m, m, k, dtype), 1, 1), ctx.mx4_quantize(normal(n, n, k, std=k ** -0.5))
    b, r = normal(k, n, dtype=dtype, std=0.3), within(normal(7, m, n, dtype=dtype), 1, 1)
    xq = ctx.mx4_quantize(x)
    xs, ws = M.held(xq), M.held(w).T
    z = xs @ ws + R.f64(b)
    off = R.sum_bound(xs, ws) + 2.0 ** -22 * np.abs(z)
    for act, save in (("none", "none"), ("gelu", "pre"), ("silu", "out"), ("relu", "none")):
        y = R.act(z, act) + R.f64(r)
        bound = R.LIPSCHITZ * off + R.ACT * (1 + np.abs(z)) + 2.0 ** -22 * np.abs(y)
        out = within(torch.zeros((m, n), dtype=dtype, device="cuda"), 1, 1)
        got = ctx.mx4_linear(x, w, b, act=act, residual=r, out=out, save=save)
        if save != "none":
            got, saved = got
            # a code is off by half a step, and by what its value was off
            step = 2.0 ** (saved.exps.cpu().numpy().astype(float)[:, np.arange(n) // 32] - 127)
            ref, ref_off = (z, off) if save == "pre" else (R.f64(got), 0.0)
            assert (np.abs(R.held(saved) - ref) <= step / 2 + ref_off + 1e-30).all()
        assert got is out and untouched(out, 1)
        R.near(got, y, bound + R.rounding(y, dtype))
        # from the 4-bit form of x, in fresh memory: the same
        again = ctx.mx4_linear(xq, w, b, act=act, residual=r, save=save)
        assert torch.equal(again if save == "none" else again[0], got)
        inplace = r.clone()
        assert torch.equal(ctx.mx4_linear(x, w, b, act=act, residual=inplace, out=inplace), got)


def test_few_tokens_share_long_sums(ctx):
    """Few weights and a long sum: the blocks of a cluster take parts of it."""
    for m, n, k in ((1, 40, 8192), (5, 65, 16384), (8, 16, 33000)):
        x, w = normal(m, m, k, dtype=torch.bfloat16), ctx.mx4_quantize(normal(n, n, k, std=k ** -0.5))
        for xx in (x, ctx.mx4_quantize(x)):
            xs, ws = M.held(ctx.mx4_quantize(x)), M.held(w).T
            got = ctx.mx4_linear(xx, w)
            R.near(got, xs @ ws, R.sum_bound(xs, ws) + R.rounding(xs @ ws, torch.bfloat16))


def test_a_nan_group_reaches_its_row_or_column_only(ctx, form):
    m, n, k = 40, 150, 600
    for rows in (m, 4):
        x, w = normal(1, rows, k, dtype=torch.bfloat16), normal(2, n, k, dtype=torch.bfloat16)
        clean = ctx.mx4_linear(x, ctx.mx4_quantize(w))
        x[2, 33], w[77, 599] = float("inf"), float("nan")
        got = ctx.mx4_linear(x, ctx.mx4_quantize(w))
        bad = torch.zeros((rows, n), dtype=torch.bool, device="cuda")
        bad[2], bad[:, 77] = True, True
        assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], clean[~bad])


def test_the_type_of_the_result(ctx):
    q, w = ctx.mx4_quantize(normal(1, 5, 64)), ctx.mx4_quantize(normal(2, 32, 64))
    assert ctx.mx4_linear(q, w).dtype == torch.bfloat16 and ctx.mx4_linear(q, w, dtype=torch.float16).dtype == torch.float16
    assert ctx.mx4_linear(q, w, torch.zeros(32, device="cuda").half()).dtype == torch.float16
    assert ctx.mx4_linear(normal(1, 5, 64).half(), w).dtype == torch.float16


# ------------------------------------------------------------------------------- gradients
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_input_grad(ctx, form, dtype, m, n, k):
    dz, w = within(varied(m, m, n, dtype), 1, 1), normal(n, n, k, std=k ** -0.5)
    wt, q = ctx.mx4_quantize_transposed(w), ctx.mx4_quantize(dz)
    a, b = M.held(q), M.held(wt).T
    r, pre = within(normal(4, m, k, dtype=dtype), 3, 1), ctx.checkpoint_save(normal(5, m, k))
    off = R.sum_bound(a, b)
    for act, residual, with_pre in (("none", None, False), ("none", r, False), ("gelu", r, True), ("relu", None, True)):
        z = R.held(pre)
        s = R.slope(z, act)
        ref = (a @ b + (0.0 if residual is None else R.f64(residual))) * s
        bound = R.LIPSCHITZ * off + (R.ACT + 2.0 ** -22) * np.abs(a @ b + (0.0 if residual is None else R.f64(residual)))
        out = within(torch.zeros((m, k), dtype=dtype, device="cuda"), 1, 1)
        sums = torch.empty(k, device="cuda")
        got, db = ctx.mx4_linear_input_grad(dz, wt, residual=residual, pre=pre if with_pre else None, act=act, out=out, bias_grad=sums)
        assert got is out and db is sums and untouched(out, 1)
        R.near(got, ref, bound + R.rounding(ref, dtype))
        R.near(db, ref.sum(axis=0), bound.sum(axis=0) + (m + 40) * 2.0 ** -24 * np.abs(ref).sum(axis=0) + 1e-30)
        again = ctx.mx4_linear_input_grad(q, wt, residual=residual, pre=pre if with_pre else None, act=act, bias_grad=False, dtype=dtype)
        assert torch.equal(again, got)
        first = sums.clone()
        ctx.mx4_linear_input_grad(q, wt, residual=residual, pre=pre if with_pre else None, act=act, bias_grad=sums, accumulate=True, dtype=dtype)
        assert torch.equal(sums, first + first)


@pytest.mark.parametrize("m,n,k", SIZES + [(2100, 70, 200), (5000, 64, 33)])
def test_weight_grad(ctx, form, m, n, k):
    dz, x = varied(m, m, n, torch.bfloat16), varied(m + 1, m, k, torch.float16)
    a, b = ctx.mx4_quantize_transposed(dz), ctx.mx4_quantize_transposed(x)
    p, q = M.held(a), M.held(b).T
    ref, off = p @ q, R.sum_bound(p, q)
    for extra, offset in ((0, 0), (1, 1), (4, 4)):
        out = within(torch.zeros((n, k), device="cuda"), extra, offset)
        got = ctx.mx4_linear_weight_grad(a, b, out=out)
        assert got is out and untouched(out, extra)
        R.near(got, ref, off + 1e-37)
        first = out.clone()
        ctx.mx4_linear_weight_grad(a, b, out=out, accumulate=True)
        assert torch.equal(out, first + first) and untouched(out, extra)
    assert torch.equal(ctx.mx4_linear_weight_grad(a, b), first)


def test_ordinary_gradients_have_no_error_at_all(ctx):
    """4-bit products whose groups are within 2^8 of one another: terms are multiples of 2^-26 of the largest
    sum's unit at most, so fp32 holds every sum of 2000 of them; a sum that lost a bit would show."""
    a, b = ctx.mx4_quantize_transposed(normal(1, 2000, 300)), ctx.mx4_quantize_transposed(normal(2, 2000, 200))
    assert np.array_equal(R.f64(ctx.mx4_linear_weight_grad(a, b)), M.held(a) @ M.held(b).T)


def test_no_tokens(ctx):
    w = ctx.mx4_quantize(normal(1, 64, 96))
    x = torch.empty((0, 96), dtype=torch.bfloat16, device="cuda")
    assert ctx.mx4_linear(x, w).shape == (0, 64) and ctx.mx4_quantize(x).codes.shape == (0, 48)
    assert ctx.mx4_linear(ctx.mx4_quantize(x), w).shape == (0, 64)
    g = torch.full((96,), 2.0, device="cuda")
    wt = ctx.mx4_quantize_transposed(normal(1, 64, 96))
    dz = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    ctx.mx4_linear_input_grad(dz, wt, bias_grad=g, accumulate=True)
    assert (g == 2).all()
    ctx.mx4_linear_input_grad(dz, wt, bias_grad=g)
    assert (g == 0).all()


def test_calls_write_their_outputs_only(ctx, form):
    for m, n, k in ((1, 33, 64), (13, 131, 300), (130, 264, 520), (300, 520, 100)):
        x, w = normal(m, m, k, dtype=torch.bfloat16), normal(n, n, k)
        out = Guarded(m, n, torch.bfloat16, 1, 1)
        ctx.mx4_linear(x, ctx.mx4_quantize(w), act="silu", out=out.view)
        out.check()
        dx, db = Guarded(m, k, torch.bfloat16, 3, 1), Guarded(1, k, torch.float32, 0, 1)
        dz = normal(m, m, n, dtype=torch.bfloat16)
        ctx.mx4_linear_input_grad(dz, ctx.mx4_quantize_transposed(w), pre=ctx.checkpoint_save(x), act="gelu", out=dx.view, bias_grad=db.view[0])
        dx.check()
        db.check()
        dw = Guarded(n, k, torch.float32, 1, 1)
        ctx.mx4_linear_weight_grad(ctx.mx4_quantize_transposed(dz), ctx.mx4_quantize_transposed(x), out=dw.view)
        dw.check()


def test_captured_and_repeated(ctx):
    """A layer's step on a stream of its own, eager and captured: the same bits; on new inputs too."""
    from paper_2108_08842_b200 import eden

    m, n, k = 300, 256, 512
    side = torch.cuda.Stream()
    c = eden.Context(0, workspace_bytes_=eden.mx4_workspace_bytes(m, n, k), stream=side)
    x, dz, w = (normal(i, *s, dtype=torch.bfloat16) for i, s in ((1, (m, k)), (2, (m, n)), (3, (n, k))))
    torch.cuda.synchronize()

    def step(c):
        rows, columns = c.mx4_quantize_both(w)
        y, pre = c.mx4_linear(x, rows, act="gelu", save="pre")
        few = c.mx4_linear(x[:3], rows)
        q, qt = c.mx4_quantize_both(dz)
        dx, db = c.mx4_linear_input_grad(q, columns, pre=c.checkpoint_save(x), act="silu")
        return [y, pre.codes, few, dx, db, c.mx4_linear_weight_grad(qt, c.mx4_quantize_transposed(x))]

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(c)
        with torch.cuda.graph(graph, stream=side):
            held = step(c)
        for seed in (1, 9):
            x.copy_(normal(seed, m, k, dtype=torch.bfloat16))
            graph.replay()
            side.synchronize()
            want = step(ctx)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))
    del graph
    assert c.status() == 0
    c.close()


def test_too_small_a_workspace_is_refused():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(1, 1, 1))
    w = c.mx4_quantize(normal(1, 64, 4096))
    with pytest.raises(eden.EdenError):
        c.mx4_linear(normal(2, 4000, 4096, dtype=torch.bfloat16), w)
    c.close()
