"""The client's training operators (linear layers, 8-bit checkpoints) against 64-bit forms."""
import numpy as np
import pytest
import torch

from tests import training_reference as R

pytestmark = pytest.mark.gpu

HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(2100, 2100, 2100))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(seed, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * std).to(dtype)


def within(t, row_extra, offset):
    """The same matrix inside a larger buffer: rows row_extra longer, `offset` elements in."""
    m, n = t.shape
    buf = torch.full((m * (n + row_extra) + offset + 1,), 7, dtype=t.dtype, device=t.device)
    v = buf[offset:offset + m * (n + row_extra)].view(m, n + row_extra)[:, :n]
    v.copy_(t)
    return v


def untouched(view, t_rows_extra):
    """Whether the gaps between the rows of a `within` view still hold the filler."""
    base, n = view._base, view.shape[1]
    full = base[view.storage_offset():view.storage_offset() + view.shape[0] * (n + t_rows_extra)].view(view.shape[0], -1)
    return bool((full[:, n:] == 7).all()) and bool((base[: view.storage_offset()] == 7).all())


# ------------------------------------------------------------------------------- checkpoints
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("m,n,extra,offset", [(1, 1, 0, 0), (3, 31, 0, 0), (2, 32, 0, 0), (5, 33, 1, 1), (7, 1000, 0, 0),
                                             (4, 1024, 0, 0), (4, 1024, 32, 3), (9, 257, 7, 2), (130, 96, 0, 0), (3, 4128, 32, 16)])
def test_checkpoint_is_the_definition(ctx, dtype, m, n, extra, offset):
    scale = torch.exp(4 * torch.randn((m, 1), generator=gen(n), device="cuda"))
    x = within((normal(n + 1, m, n) * scale).to(dtype), extra, offset)
    saved = ctx.checkpoint_save(x)
    codes, exps = R.code(R.f64(x))
    assert np.array_equal(saved.codes.cpu().numpy(), codes) and np.array_equal(saved.exps.cpu().numpy(), exps)
    back = ctx.checkpoint_restore(saved, dtype)
    R.near(back, R.restored(codes, exps, dtype), R.TINY[dtype] if dtype == torch.float16 else 0.0)   # exact, fp16 below 2^-24 rounds
    step = 2.0 ** (exps[:, np.arange(n) // 32] - 127.0)
    with np.errstate(invalid="ignore"):
        near = np.abs(R.f64(back) - R.f64(x)) <= step / 2 + (R.TINY[dtype] if dtype == torch.float16 else 0)
    assert (near | (exps[:, np.arange(n) // 32] == 255)).all()


@pytest.mark.parametrize("offset", [0, 1])
def test_checkpoint_into_views(ctx, offset):
    m, n = 6, 320
    x = normal(3, m, n, dtype=torch.bfloat16)
    plain = ctx.checkpoint_save(x)
    out = (within(torch.zeros((m, n), dtype=torch.int8, device="cuda"), 32 + offset, 32 + offset),
           within(torch.zeros((m, n // 32), dtype=torch.uint8, device="cuda"), 3, offset))
    ctx.checkpoint_save(x, out)
    assert torch.equal(out[0], plain.codes) and torch.equal(out[1], plain.exps)
    assert untouched(out[0], 32 + offset) and untouched(out[1], 3)
    y = within(torch.zeros_like(x), 16 + offset, 16 + offset)
    ctx.checkpoint_restore(out, torch.bfloat16, y)
    assert torch.equal(y, ctx.checkpoint_restore(plain, torch.bfloat16)) and untouched(y, 16 + offset)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_checkpoint_of_special_values(ctx, dtype):
    top = torch.finfo(dtype).max
    small = torch.finfo(dtype).smallest_normal
    rows = [[0.0] * 40, [-0.0] * 40, [top, -top, 1.0] + [0.0] * 37, [small, -small * 0.5] + [0.0] * 38,
            [127.0, 126.5, -125.5, 0.5, 1.5, 2.5] + [0.0] * 34, [127.5] + [1.0] * 39, [1.0] * 32 + [1e-3] * 8,
            [float("inf")] + [1.0] * 39, [float("nan")] + [2.0] * 39, [1.0] * 39 + [float("-inf")], [1.0] * 32 + [float("nan")] * 8,
            [63.5, 127.0 / 64, 128.0 / 64] + [0.0] * 37]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype).cuda()
    saved = ctx.checkpoint_save(x)
    codes, exps = R.code(R.f64(x))
    assert np.array_equal(saved.codes.cpu().numpy(), codes) and np.array_equal(saved.exps.cpu().numpy(), exps)
    R.near(ctx.checkpoint_restore(saved, dtype), R.restored(codes, exps, dtype), R.TINY[dtype])


def test_checkpoint_restores_any_codes_and_exponents(ctx):
    # what another program wrote: every code, exponents over the whole range
    codes = torch.arange(-128, 128, device="cuda").to(torch.int8).repeat(8, 1).contiguous()
    exps = torch.arange(64, device="cuda").mul(4).add(1).to(torch.uint8).view(8, 8)
    exps[7, 7] = 255
    ref = R.restored(codes.cpu().numpy(), exps.cpu().numpy().astype(np.int64), torch.float32)
    R.near(ctx.checkpoint_restore((codes, exps), torch.float32), ref, 0.0)


# ------------------------------------------------------------------------------- forward
def check_linear(ctx, dtype, m, n, k, act, with_bias, with_residual, save, extra=0, offset=0, seed=0):
    x = within(normal(seed + 1, m, k, dtype=dtype), extra, offset)
    w = within(normal(seed + 2, n, k, dtype=dtype, std=k ** -0.5), extra, offset)
    b = normal(seed + 3, n, dtype=dtype, std=0.3) if with_bias else None
    r = within(normal(seed + 4, m, n, dtype=dtype), extra, offset) if with_residual else None
    out = within(torch.zeros((m, n), dtype=dtype, device="cuda"), extra, offset)
    got = ctx.linear(x, w, b, act=act, residual=r, out=out, save=save)
    saved = None
    if save != "none":
        got, saved = got
    assert got is out and untouched(out, extra)
    xs, ws = R.f64(x), R.f64(w).T
    z = xs @ ws + (R.f64(b) if with_bias else 0.0)
    off = R.sum_bound(xs, ws) + 2.0 ** -22 * np.abs(z)
    y = R.act(z, act) + (R.f64(r) if with_residual else 0.0)
    bound = R.LIPSCHITZ * off + R.ACT * (1 + np.abs(z)) + 2.0 ** -23 * np.abs(y)
    R.near(got, y, bound + R.rounding(np.abs(y) + bound, dtype))
    if save == "out":
        again = ctx.checkpoint_save(out)
        assert torch.equal(saved.codes, again.codes) and torch.equal(saved.exps, again.exps)
    if save == "pre":
        e = saved.exps.cpu().numpy().astype(float)[:, np.arange(n) // 32] - 127
        assert (np.abs(R.held(saved) - z) <= 2.0 ** e / 2 + off).all()
        top = np.stack([np.abs(z)[:, g:g + 32].max(axis=1) for g in range(0, n, 32)], axis=1)[:, np.arange(n) // 32]
        slack = np.stack([off[:, g:g + 32].max(axis=1) for g in range(0, n, 32)], axis=1)[:, np.arange(n) // 32]
        assert (top - slack <= 127 * 2.0 ** e).all() and (top + slack > 127 * 2.0 ** (e - 1)).all()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 64), (1, 4096, 1024), (2, 33, 7), (5, 1000, 1000), (8, 512, 2048), (9, 96, 72),
                                   (13, 2731, 1000), (16, 2048, 136), (17, 130, 40), (32, 640, 512), (33, 257, 129), (64, 1024, 1024),
                                   (100, 300, 200), (127, 128, 64), (128, 256, 192), (129, 255, 65), (256, 256, 64), (257, 513, 264),
                                   (300, 1024, 1000), (511, 96, 2056), (1000, 768, 320)])
def test_linear_sizes(ctx, dtype, m, n, k):
    check_linear(ctx, dtype, m, n, k, "none", True, True, "none", seed=m + n + k)


@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("m,n,k", [(1, 160, 256), (37, 96, 64), (200, 544, 128)])
@pytest.mark.parametrize("save", ["none", "pre", "out"])
def test_linear_activations_and_saves(ctx, act, m, n, k, save):
    check_linear(ctx, torch.bfloat16, m, n, k, act, True, save == "out", save, seed=m)
    check_linear(ctx, torch.float16, m, n + 5, k, act, False, True, save, seed=m)


@pytest.mark.parametrize("extra,offset", [(1, 0), (8, 8), (3, 5), (16, 16), (8, 1), (0, 2)])
@pytest.mark.parametrize("m,n,k", [(1, 96, 128), (7, 72, 128), (70, 200, 128), (260, 384, 136)])
def test_linear_strides_and_alignment(ctx, extra, offset, m, n, k):
    check_linear(ctx, torch.bfloat16, m, n, k, "silu", True, True, "pre", extra, offset)


@pytest.mark.parametrize("m", [1, 9, 200])
def test_linear_residual_in_place(ctx, m):
    x, w = normal(1, m, 256, dtype=torch.bfloat16), normal(2, 320, 256, dtype=torch.bfloat16, std=0.06)
    r = normal(3, m, 320, dtype=torch.bfloat16)
    want = ctx.linear(x, w, residual=r)
    ctx.linear(x, w, residual=r, out=r)
    assert torch.equal(want, r)


@pytest.mark.parametrize("m", [1, 12, 300])
def test_linear_rows_do_not_meet(ctx, m):
    """A row of infinities and a row of NaN leave the other rows as they are."""
    x, w = normal(1, m + 2, 192, dtype=torch.bfloat16), normal(2, 288, 192, dtype=torch.bfloat16, std=0.07)
    b = normal(3, 288, dtype=torch.bfloat16)
    want, kept = ctx.linear(x, w, b, act="relu", save="pre")
    x[m // 2] = float("inf")
    x[m + 1] = float("nan")
    got, saved = ctx.linear(x, w, b, act="relu", save="pre")
    others = [i for i in range(m + 2) if i not in (m // 2, m + 1)]
    assert torch.equal(got[others], want[others]) and torch.equal(saved.codes[others], kept.codes[others])
    assert not torch.isfinite(got[m + 1]).any() and (saved.exps[m + 1] == 255).all() and (saved.exps[m // 2] == 255).all()
    assert torch.isnan(ctx.checkpoint_restore(saved, torch.bfloat16)[m + 1]).all()


def test_linear_fp16_overflow_is_infinite(ctx):
    for m in (1, 40):
        x = torch.full((m, 64), 200.0, dtype=torch.float16, device="cuda")
        y, saved = ctx.linear(x, torch.full((32, 64), 200.0, dtype=torch.float16, device="cuda"), save="pre")
        assert (y == float("inf")).all()                       # 64 * 40000 is past fp16's largest
        assert (np.abs(R.held(saved) - 64 * 40000.0) <= 2.0 ** 15 / 2).all()     # 2560000 lies between 127 * 2^14 and 127 * 2^15


def test_linear_of_no_tokens(ctx):
    w = normal(2, 48, 64, dtype=torch.bfloat16)
    y, saved = ctx.linear(normal(1, 0, 64, dtype=torch.bfloat16), w, save="out")
    assert y.shape == (0, 48) and saved.codes.shape == (0, 48)
    dx, db = ctx.linear_input_grad(normal(1, 0, 48, dtype=torch.bfloat16), w, pre=ctx.checkpoint_empty(0, 64), act="gelu")
    assert dx.shape == (0, 64) and torch.equal(db, torch.zeros(64, device="cuda"))
    dw = ctx.linear_weight_grad(normal(1, 0, 48, dtype=torch.bfloat16), normal(1, 0, 64, dtype=torch.bfloat16))
    assert torch.equal(dw, torch.zeros((48, 64), device="cuda"))
    dw.fill_(3)
    ctx.linear_weight_grad(normal(1, 0, 48, dtype=torch.bfloat16), ctx.checkpoint_empty(0, 64), out=dw, accumulate=True)
    assert (dw == 3).all()
    dz, db = ctx.act_backward(normal(1, 0, 48, dtype=torch.bfloat16), ctx.checkpoint_empty(0, 48), act="silu")
    assert dz.shape == (0, 48) and torch.equal(db, torch.zeros(48, device="cuda"))
    assert ctx.checkpoint_restore(ctx.checkpoint_save(normal(1, 0, 5)), torch.float32).shape == (0, 5)


FORMS = [(f, s) for f in ("LINEAR_PAIR", "LINEAR_SINGLE", "LINEAR_NARROW") for s in (1, 2, 4, 8)]


@pytest.fixture
def forced(ctx, request):
    from paper_2108_08842_b200 import eden

    form, splits = request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, getattr(eden, form))
    ctx.set_option(eden.OPT_LINEAR_SPLITS, splits)
    yield request.param
    ctx.set_option(eden.OPT_LINEAR_FORM, eden.LINEAR_AUTO)
    ctx.set_option(eden.OPT_LINEAR_SPLITS, 0)


@pytest.mark.parametrize("forced", FORMS, indirect=True)
def test_every_form_at_every_size(ctx, forced):
    """Each kernel form, with each number of parts, on sizes that the choice would give another."""
    for m, n, k in ((1, 40, 72), (48, 1000, 520), (200, 300, 1000), (520, 264, 64), (300, 700, 520)):
        check_linear(ctx, torch.bfloat16, m, n, k, "silu", True, True, "pre", seed=m)
        check_input_grad(ctx, torch.float16, m, n, k, "gelu", True)
        check_weight_grad(ctx, torch.bfloat16, m, n, k, True)
    check_linear(ctx, torch.float16, 150, 333, 777, "relu", True, True, "out", 3, 1)
    check_weight_grad(ctx, torch.float16, 1111, 130, 270, False, 1, 1)


def test_last_wave_in_parts():
    """80 tiles of 256 x 256 on 74 pairs of SMs: the rest of the tiles in a launch of their own."""
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(4096, 4096, 4096))
    x, w = normal(1, 1270, 4096, dtype=torch.bfloat16), normal(2, 4000, 4096, dtype=torch.bfloat16, std=0.015)
    b, r = normal(3, 4000, dtype=torch.bfloat16), normal(4, 1270, 4000, dtype=torch.bfloat16)
    before = c.launch_count
    y, saved = c.linear(x, w, b, act="silu", residual=r, save="pre")
    assert c.launch_count == before + 2
    c.set_option(eden.OPT_LINEAR_SPLITS, 1)
    plain = c.linear(x, w, b, act="silu", residual=r)
    assert c.launch_count == before + 3
    c.set_option(eden.OPT_LINEAR_SPLITS, 0)
    xs, ws = R.f64(x), R.f64(w).T
    z = xs @ ws + R.f64(b)
    off = R.sum_bound(xs, ws) + 2.0 ** -22 * np.abs(z)
    ref = R.act(z, "silu") + R.f64(r)
    bound = R.LIPSCHITZ * off + R.ACT * (1 + np.abs(z)) + 2.0 ** -23 * np.abs(ref)
    for got in (y, plain):
        R.near(got, ref, bound + R.rounding(np.abs(ref) + bound, torch.bfloat16))
    step = 2.0 ** (saved.exps.cpu().numpy().astype(float)[:, np.arange(4000) // 32] - 127)
    assert (np.abs(R.held(saved) - z) <= step / 2 + off).all()
    # sums over 4096 tokens into 80 tiles
    before = c.launch_count
    dw = c.linear_weight_grad(x.t().contiguous(), w.t().contiguous())
    assert c.launch_count == before + 3                # rows of 1270 values are laid out first
    R.near(dw, xs @ ws, R.sum_bound(xs, ws))
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("forced", [("LINEAR_FEW", 0)], indirect=True)
@pytest.mark.parametrize("m,n,k,extra,offset", [(17, 100, 1000, 0, 0), (24, 33, 4104, 8, 8), (31, 64, 200, 1, 1), (32, 16, 5000, 0, 0), (33, 64, 64, 0, 0)])
def test_few_tokens_form(ctx, forced, m, n, k, extra, offset):
    for save in ("none", "pre", "out"):
        check_linear(ctx, torch.bfloat16, m, n, k, "gelu_tanh", True, True, save, extra, offset)


@pytest.mark.parametrize("offset", range(8))
@pytest.mark.parametrize("m,k", [(1, 1001), (2, 1002), (3, 517), (9, 1028), (12, 71), (40, 333), (40, 334)])
def test_linear_rows_at_every_alignment(ctx, m, k, offset):
    check_linear(ctx, torch.float16, m, 50, k, "none", True, False, "pre" if offset % 2 else "none", 0, offset, seed=k)


# ------------------------------------------------------------------------------- backward
def pre_of(seed, m, n):
    codes, exps = R.code(R.f64(normal(seed, m, n, std=2.0)))
    return torch.from_numpy(codes.astype(np.int8)).cuda(), torch.from_numpy(exps.astype(np.uint8)).cuda()


def column_bound(d, off):
    """fp32 column sums of values that are off by `off` each."""
    return (d.shape[0] + 8) * 2.0 ** -23 * np.abs(d).sum(axis=0) + off.sum(axis=0)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("m,n,extra,offset", [(1, 1, 0, 0), (1, 4096, 0, 0), (3, 33, 0, 0), (64, 256, 0, 0), (333, 999, 0, 0),
                                             (200, 128, 32, 5), (1030, 64, 32, 32), (65, 2080, 16, 16)])
def test_act_backward(ctx, dtype, act, m, n, extra, offset):
    dy = within(normal(m, m, n, dtype=dtype, std=0.02), extra, offset)
    pre = tuple(within(t, extra, offset) for t in pre_of(n, m, n))
    out = within(torch.zeros((m, n), dtype=dtype, device="cuda"), extra, offset)
    dz, db = ctx.act_backward(dy, pre, act=act, out=out)
    z = R.held(pre)
    ref = R.f64(dy) * R.slope(z, act)
    off = np.abs(R.f64(dy)) * R.ACT
    R.near(dz, ref, off + R.rounding(np.abs(ref) + off, dtype))
    R.near(db, ref.sum(axis=0), column_bound(ref, off))
    assert untouched(out, extra)
    twice = db.clone()
    ctx.act_backward(dy, pre, act=act, out=out, bias_grad=twice, accumulate=True)
    R.near(twice, R.f64(db) * 2, 2.0 ** -22 * np.abs(R.f64(db)))
    assert torch.equal(out, dz)
    own = dy.clone()
    ctx.act_backward(own, pre, act=act, out=own)               # in place
    assert torch.equal(own, dz)


def test_act_slopes_are_the_differences(ctx):
    """dz / dy against central differences of the activation in 64 bits."""
    codes = torch.arange(-127, 128, device="cuda").to(torch.int8).repeat(9, 1).contiguous()
    exps = (torch.arange(-9, 0, device="cuda") + 2 + 127).to(torch.uint8)[:, None].repeat(1, 8).contiguous()   # |z| up to 127
    dy = torch.ones((9, 255), dtype=torch.float16, device="cuda")
    z = R.held((codes, exps))
    h = 1e-6
    for act in R.ACTS:
        dz, _ = ctx.act_backward(dy, (codes, exps), act=act)
        diff = (R.act(z + h, act) - R.act(z - h, act)) / (2 * h)
        live = (np.abs(z) > 2 * h) if act == "relu" else np.ones_like(z, bool)
        # the differences: third derivatives below 4, 64-bit rounding of values up to 127
        bound = 4 * h * h + 127 * 2.0 ** -52 / h + R.ACT
        assert (np.abs(R.f64(dz) - diff) <= bound + R.rounding(np.abs(diff) + bound, torch.float16))[live].all(), act
    dz, _ = ctx.act_backward(dy, (codes, exps), act="relu")
    assert (R.f64(dz)[z == 0] == 0).all()


def test_act_backward_extremes(ctx):
    """Saturated, empty and NaN groups."""
    codes = torch.tensor([[-127, 127, 0, 1]], dtype=torch.int8, device="cuda").repeat(4, 1)
    exps = torch.tensor([[248], [1], [140], [255]], dtype=torch.uint8, device="cuda")
    codes[3] = 0
    dy = torch.full((4, 4), 2.0, dtype=torch.bfloat16, device="cuda")
    for act in R.ACTS[1:]:
        dz, _ = ctx.act_backward(dy, (codes, exps), act=act)
        got = R.f64(dz)
        assert np.isnan(got[3]).all()
        assert np.array_equal(got[0, :2], [0, 2]) and np.array_equal(got[2, :2], [0, 2]), act
        assert np.array_equal(got[1], [0, 2, 0, 2] if act == "relu" else [1, 1, 1, 1])


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 512, 256), (2, 7, 33), (16, 136, 200), (33, 129, 257), (64, 512, 1024), (100, 200, 300),
                                   (128, 64, 256), (129, 65, 255), (300, 1000, 1024), (517, 264, 520), (1000, 320, 768)])
@pytest.mark.parametrize("act,residual", [(None, False), (None, True), ("gelu", False), ("relu", True)])
def test_input_grad(ctx, dtype, m, n, k, act, residual):
    check_input_grad(ctx, dtype, m, n, k, act, residual)


@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("m,n,k,extra,offset", [(5, 40, 72, 1, 1), (70, 128, 200, 8, 8), (260, 136, 384, 16, 16), (260, 136, 384, 3, 5)])
def test_input_grad_strides(ctx, act, m, n, k, extra, offset):
    check_input_grad(ctx, torch.bfloat16, m, n, k, act, True, extra, offset)


def check_input_grad(ctx, dtype, m, n, k, act, residual, extra=0, offset=0):
    dz = within(normal(m, m, n, dtype=dtype, std=0.02), extra, offset)
    w = within(normal(n, n, k, dtype=dtype, std=n ** -0.5), extra, offset)
    r = within(normal(k, m, k, dtype=dtype, std=0.02), extra, offset) if residual else None
    out = within(torch.zeros((m, k), dtype=dtype, device="cuda"), extra, offset)
    pre = None if act is None else tuple(within(t, extra, offset) for t in pre_of(m + k, m, k))
    got = ctx.linear_input_grad(dz, w, residual=r, pre=pre, act=act or "none", out=out)
    assert untouched(out, extra)
    a, b = R.f64(dz), R.f64(w)
    inner = a @ b + (R.f64(r) if residual else 0.0)
    off = R.sum_bound(a, b) + 2.0 ** -23 * np.abs(inner)
    if act is None:
        return R.near(got, inner, off + R.rounding(np.abs(inner) + off, dtype))
    dx, db = got
    s = R.slope(R.held(pre), act)
    ref = inner * s
    off = off * R.LIPSCHITZ + np.abs(inner) * R.ACT
    R.near(dx, ref, off + R.rounding(np.abs(ref) + off, dtype))
    R.near(db, ref.sum(axis=0), column_bound(ref, off))
    base = torch.full_like(db, 0.5)
    ctx.linear_input_grad(dz, w, residual=r, pre=pre, act=act, out=out, bias_grad=base, accumulate=True)
    R.near(base, R.f64(db) + 0.5, 2.0 ** -23 * (np.abs(R.f64(db)) + 0.5))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 96), (3, 33, 7), (31, 128, 128), (64, 256, 256), (65, 100, 300), (100, 257, 129),
                                   (500, 136, 200), (1000, 512, 256), (2050, 96, 64), (129, 1000, 1024)])
@pytest.mark.parametrize("held", [True, False])
def test_weight_grad(ctx, dtype, m, n, k, held):
    check_weight_grad(ctx, dtype, m, n, k, held)


@pytest.mark.parametrize("held", [True, False])
@pytest.mark.parametrize("m,n,k,extra,offset", [(40, 72, 33, 1, 1), (130, 200, 264, 8, 8), (130, 200, 256, 16, 16), (300, 260, 384, 3, 5)])
def test_weight_grad_strides(ctx, held, m, n, k, extra, offset):
    check_weight_grad(ctx, torch.bfloat16, m, n, k, held, extra, offset)


def check_weight_grad(ctx, dtype, m, n, k, held, extra=0, offset=0):
    dz = within(normal(m, m, n, dtype=dtype, std=0.02), extra, offset)
    if held:
        x = tuple(within(t, extra, offset) for t in pre_of(m + k, m, k))
        xs = R.held(x)
    else:
        x = within(normal(m + k, m, k, dtype=dtype), extra, offset)
        xs = R.f64(x)
    out = within(torch.zeros((n, k), device="cuda"), extra, offset)
    ctx.linear_weight_grad(dz, x, out=out)
    assert untouched(out, extra)
    a = R.f64(dz).T
    ref, off = a @ xs, R.sum_bound(a, xs)
    R.near(out, ref, off)
    before = R.f64(out)
    ctx.linear_weight_grad(dz, x, out=out, accumulate=True)
    R.near(out, before + ref, off + 2.0 ** -23 * np.abs(before + ref) * (1 + 1e-6))


def test_products_are_the_differences_of_the_forward(ctx):
    """<dy, act(x W^T + b)> in 64 bits, differenced at entries of x, W and b: what the chain
    act_backward, input_grad, weight_grad returns for it."""
    m, n, k, act = 24, 40, 48, "gelu"
    x, w = normal(1, m, k, dtype=torch.float16), normal(2, n, k, dtype=torch.float16, std=0.15)
    b, dy = normal(3, n, dtype=torch.float16, std=0.2), normal(4, m, n, dtype=torch.float16)
    _, pre = ctx.linear(x, w, b, act=act, save="pre")
    saved = ctx.checkpoint_save(x)
    dz, db = ctx.act_backward(dy, pre, act=act)
    dx, dw = ctx.linear_input_grad(dz, w), ctx.linear_weight_grad(dz, saved)
    xs, ws, bs, ds = R.f64(x), R.f64(w), R.f64(b), R.f64(dy)
    zq, xq = R.held(pre), R.held(saved)

    def loss(xv, wv, bv, at):
        # the backward pass sees the checkpointed pre-activation: differences are taken around it
        return (ds * R.act(zq + (xv @ wv.T + bv) - at, act)).sum()

    h = 1e-5
    at = xs @ ws.T + bs
    rng = np.random.default_rng(0)
    grain = 2.0 ** -11 * np.abs(ds).max() * R.LIPSCHITZ * 1.01 + R.ACT * np.abs(ds).max()    # dz: fp16, below 8
    for _ in range(12):
        i, j, c = rng.integers(m), rng.integers(n), rng.integers(k)
        e = np.zeros_like(xs); e[i, c] = h
        diff = (loss(xs + e, ws, bs, at) - loss(xs - e, ws, bs, at)) / (2 * h)
        assert abs(R.f64(dx)[i, c] - diff) <= grain * np.abs(ws[:, c]).sum() + 2.0 ** -10 * abs(diff) + 1e-6
        e = np.zeros_like(bs); e[j] = h
        diff = (loss(xs, ws, bs + e, at) - loss(xs, ws, bs - e, at)) / (2 * h)
        assert abs(R.f64(db)[j] - diff) <= m * R.ACT * np.abs(ds).max() + 1e-6
        # the weight's gradient reads the checkpointed input
        e = np.zeros_like(ws); e[j, c] = h
        at_q = xq @ ws.T + bs
        diff = (loss(xq, ws + e, bs, at_q) - loss(xq, ws - e, bs, at_q)) / (2 * h)
        assert abs(R.f64(dw)[j, c] - diff) <= grain * np.abs(xq[:, c]).sum() + 1e-6


def test_results_repeat_bit_for_bit(ctx):
    x, w = normal(1, 700, 1024, dtype=torch.bfloat16), normal(2, 640, 1024, dtype=torch.bfloat16)
    pre = pre_of(3, 700, 1024)
    dz = normal(4, 700, 640, dtype=torch.bfloat16)
    first = None
    for _ in range(3):
        got = [ctx.linear(x, w), *ctx.linear_input_grad(dz, w, pre=pre, act="silu"), ctx.linear_weight_grad(dz, pre),
               *ctx.act_backward(x, pre, act="gelu"), ctx.linear(x[:3], w)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


# ------------------------------------------------------------------------------- use
def test_calls_on_another_stream(ctx):
    from paper_2108_08842_b200 import eden

    side = torch.cuda.Stream()
    other = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(512, 512, 512), stream=side)
    x, w = normal(1, 500, 512, dtype=torch.bfloat16), normal(2, 512, 512, dtype=torch.bfloat16, std=0.05)
    want = ctx.linear(x, w, act="gelu")
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):                                # inputs freed by the caller at once
        xs = x.clone()
        side.wait_stream(torch.cuda.current_stream())
        y, saved = other.linear(xs, w, act="gelu", save="out")
        del xs
        junk = torch.full_like(x, float("nan"))
        z = other.checkpoint_restore(saved, torch.bfloat16)
        del junk
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want) and torch.equal(z, ctx.checkpoint_restore(ctx.checkpoint_save(want), torch.bfloat16))
    torch.cuda.synchronize()
    assert other.status() == 0
    other.close()


def test_offsets_past_32_bits(ctx):
    """Matrices of more than 2^31 elements, and rows further apart than that in all."""
    m, n = 70000, 32768
    x = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    x.copy_(torch.arange(n, device="cuda").sub(n // 2).mul(2.0 ** -10).to(torch.bfloat16).expand(m, n))
    x[-1] = x[-1].flip(0)
    saved = ctx.checkpoint_save(x)
    back = ctx.checkpoint_restore(saved, torch.bfloat16)
    for r in (0, 40000, m - 1):
        codes, exps = R.code(R.f64(x[r:r + 1]))
        assert np.array_equal(saved.codes[r:r + 1].cpu().numpy(), codes) and np.array_equal(saved.exps[r:r + 1].cpu().numpy(), exps)
        R.near(back[r:r + 1], R.value(codes, exps), 0.0)
    dz, db = ctx.act_backward(x[-600:], (saved.codes[-600:], saved.exps[-600:]), act="relu", out=back[-600:])
    z = R.held((saved.codes[-600:], saved.exps[-600:]))
    R.near(dz, R.f64(x[-600:]) * (z > 0), R.rounding(R.f64(x[-600:]), torch.bfloat16))
    del back, saved, dz
    # 300 rows, 2^23 elements apart
    step, k = 1 << 23, 200
    wide = x.view(-1).as_strided((270, k), (step, 1))
    assert wide.numel() == 270 * k and 269 * step > 2 ** 31
    wide.copy_(normal(1, 270, k, dtype=torch.bfloat16))
    w = normal(2, 96, k, dtype=torch.bfloat16, std=0.07)
    xs, ws = R.f64(wide), R.f64(w).T
    off = R.sum_bound(xs, ws)
    out = x.view(-1).as_strided((270, 96), (step, 1), storage_offset=1024)
    R.near(ctx.linear(wide, w, out=out), xs @ ws, off + R.rounding(np.abs(xs @ ws) + off, torch.bfloat16))
    R.near(ctx.linear(wide[-3:], w, out=out[-3:]), (xs @ ws)[-3:], (off + R.rounding(np.abs(xs @ ws) + off, torch.bfloat16))[-3:])
    ref = R.f64(out).T @ xs
    R.near(ctx.linear_weight_grad(out, wide), ref, R.sum_bound(R.f64(out).T, xs))


def test_two_contexts_at_once(ctx):
    """Products on two streams whose kernels want the same SMs and tensor memory."""
    from paper_2108_08842_b200 import eden

    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(600, 1024, 1024), stream=s) for s in streams]
    x, w = normal(1, 600, 1024, dtype=torch.bfloat16), normal(2, 1024, 1024, dtype=torch.bfloat16, std=0.03)
    pre = pre_of(3, 600, 1024)
    want = ctx.linear(x, w, act="gelu"), ctx.linear_weight_grad(x, pre), ctx.linear(x[:5], w)
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for c in both:
            got.append((c.linear(x, w, act="gelu"), c.linear_weight_grad(x, pre), c.linear(x[:5], w)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
    for c in both:
        assert c.status() == 0
        c.close()


def test_calls_in_a_graph():
    from paper_2108_08842_b200 import eden

    side = torch.cuda.Stream()
    c = eden.Context(0, workspace_bytes_=eden.linear_workspace_bytes(300, 256, 1000), stream=side)
    x, w = normal(1, 300, 1000, dtype=torch.bfloat16), normal(2, 256, 1000, dtype=torch.bfloat16, std=0.03)
    y, dw, saved = torch.empty((300, 256), dtype=torch.bfloat16, device="cuda"), torch.empty((256, 1000), device="cuda"), c.checkpoint_empty(300, 1000)

    def step():
        c.linear(x, w, act="silu", out=y)
        c.checkpoint_save(x, saved)
        c.linear_weight_grad(y, saved, out=dw)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    got = y.clone(), dw.clone()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert torch.equal(got[0], y) and torch.equal(got[1], dw)
    assert c.status() == 0
    c.close()


def test_training_calls_between_encode_and_mean():
    """The calls share the context's workspace with the sender and the receiver."""
    from paper_2108_08842_b200 import eden

    d, n = 1 << 16, 3
    c = eden.Context(0, workspace_bytes_=max(eden.workspace_bytes(d, n), eden.linear_workspace_bytes(256, 256, 256)))
    x = normal(1, n, d)
    bits, seeds = [1.0, 0.5, 4.0], [3, 4, 5]
    codes, scales = c.encode(x, bits, seeds)
    want = c.mean(codes, scales, bits, seeds, d)
    codes2, scales2 = c.encode(x, bits, seeds)
    c.linear_weight_grad(normal(2, 256, 256, dtype=torch.bfloat16), c.checkpoint_save(normal(3, 256, 256, dtype=torch.bfloat16)))
    with pytest.raises(eden.EdenError):
        c.client_stats(n)                              # gone, and said so
    got = c.mean(codes2, scales2, bits, seeds, d)
    assert torch.equal(want, got) and len(c.client_stats(n)) == n and c.status() == 0
    c.close()


def test_refusals(ctx):
    from paper_2108_08842_b200 import eden

    x, w = normal(1, 8, 64, dtype=torch.bfloat16), normal(2, 32, 64, dtype=torch.bfloat16)
    ck = ctx.checkpoint_save(x)
    for bad in (lambda: ctx.linear(x.float(), w), lambda: ctx.linear(x.float(), w.float()), lambda: ctx.linear(x, w.half()),
                lambda: ctx.linear(x, w[:, :60]), lambda: ctx.linear(x.cpu(), w), lambda: ctx.linear(x[0], w),
                lambda: ctx.linear(x, w.t().contiguous().t()), lambda: ctx.linear(x, w, act="tanh"), lambda: ctx.linear(x, w, save="all"),
                lambda: ctx.linear(x, w, bias=normal(1, 31, dtype=torch.bfloat16)), lambda: ctx.linear(x, w, bias=normal(1, 32)),
                lambda: ctx.linear(x, w, residual=x), lambda: ctx.linear(x, w, out=normal(1, 8, 32)),
                lambda: ctx.linear(x[:1].expand(8, 64), w), lambda: ctx.linear(x, w, save="pre", saved=ck),
                lambda: ctx.checkpoint_save(x.double()), lambda: ctx.checkpoint_restore(ck, torch.int8),
                lambda: ctx.checkpoint_restore((ck[0], ck[1][:, :1]), torch.bfloat16), lambda: ctx.act_backward(x, None, act="gelu"),
                lambda: ctx.act_backward(x, ck, act="gelu", accumulate=True), lambda: ctx.act_backward(x[:, :32], ck, act="gelu"),
                lambda: ctx.linear_input_grad(x[:, :32], w, act="gelu"), lambda: ctx.linear_input_grad(x, w),
                lambda: ctx.linear_weight_grad(x, ck, accumulate=True), lambda: ctx.linear_weight_grad(x, x.half()),
                lambda: ctx.linear_weight_grad(x, ck, out=normal(1, 64, 64, dtype=torch.bfloat16))):
        with pytest.raises((ValueError, eden.EdenError)):
            bad()
    for shape in ((8, 0), (0, 0)):
        with pytest.raises(eden.EdenError):
            ctx.checkpoint_save(torch.empty(shape, device="cuda"))
    small = eden.Context(0, workspace_bytes_=1 << 20)
    with pytest.raises(eden.EdenError) as e:
        small.linear_weight_grad(normal(1, 2048, 64, dtype=torch.bfloat16), ctx.checkpoint_save(normal(2, 2048, 1024, dtype=torch.bfloat16)))
    assert e.value.code == -4
    assert small.status() == 0
    small.close()
