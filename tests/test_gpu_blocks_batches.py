"""Joins of more rows than a launch has places for: a team, or a cluster, takes several rows one after the
other, so that the places that its rows are brought to, and those of its sums, are used again."""
import pytest
import torch

from tests import test_gpu_blocks as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2108_08842_b200 import eden

    c = eden.Context(0, workspace_bytes_=eden.block_workspace_bytes(32768))
    yield c
    torch.cuda.synchronize()
    assert c.status() == 0
    c.close()


BOTH = [("rms", "rms", "vector", True, 0.25), ("layer", "layer", "matrix", True, 0.1)]


# 37 or 74 clusters of 4 or 2 blocks: 3 to 6 rows each, in 2 to 4 places
@pytest.mark.parametrize("parts", BOTH, ids=lambda p: "-".join(map(str, p)))
@pytest.mark.parametrize("m,n,extra,offset,held", [(400, 8200, 0, 0, True), (400, 8200, 1, 1, False), (100, 16390, 0, 0, True), (120, 32768, 0, 0, False)])
def test_clusters_take_several_rows(ctx, parts, m, n, extra, offset, held):
    T.check_join(ctx, T.Case(m, n, torch.bfloat16, *parts, bias=n % 2 == 0, extra=extra, offset=offset))
    T.test_join_backward(ctx, torch.bfloat16, *parts, m, n, extra, offset, held)


# teams of a warp to all of a block's, of one piece a thread and of two, aligned rows and others: 4 to 16 rows a
# team, in 2 to 4 places
@pytest.mark.parametrize("parts", BOTH + [("rms", "none", "matrix", True, 0.3), ("none", "layer", "vector", False, 0.0)], ids=lambda p: "-".join(map(str, p)))
@pytest.mark.parametrize("m,n,extra,offset,held", [(30000, 40, 0, 0, True), (8000, 513, 0, 0, False), (1600, 4096, 0, 0, True), (1200, 4104, 8, 8, False)])
def test_teams_take_several_rows(ctx, parts, m, n, extra, offset, held):
    T.check_join(ctx, T.Case(m, n, torch.bfloat16, *parts, bias=n % 2 == 0, extra=extra, offset=offset))
    T.test_join_backward(ctx, torch.bfloat16, *parts, m, n, extra, offset, held)


def test_a_batch_is_its_rows(ctx):
    """The rows of a batch, joined in parts of one row a team, are the same bit for bit, forward and backward."""
    m, n, part = 8000, 520, 800
    c = T.Case(m, n, torch.float16, "layer", "rms", "vector", drop=0.2, bias=True)
    j = ctx.block_join(c.h, c.residual, stats=True, **c.how())
    dx, dy = T.make(5, m, n, torch.float16), T.make(6, m, n, torch.float16)
    sums = dict(after_bias_grad=False, before_bias_grad=False)        # which would have the parts take fewer values a thread
    d = ctx.block_join_backward(dx, dy, c.h, j.x, j.after_stats, j.before_stats, **sums, **c.how())
    for i in range(0, m, part):
        s, how = slice(i, i + part), {**c.how(), "first_row": i}
        a = ctx.block_join(c.h[s], c.residual[s], stats=True, **how)
        assert all(torch.equal(p, q[s]) for p, q in zip(a, j))
        b = ctx.block_join_backward(dx[s], dy[s], c.h[s], j.x[s], j.after_stats[s], j.before_stats[s], **sums, **how)
        assert torch.equal(b.h, d.h[s]) and torch.equal(b.residual, d.residual[s])


# rows that the first seven blocks of a cluster hold
@pytest.mark.parametrize("m,n,extra,offset,parts", [(40, 20488, 0, 0, ("layer", "layer", "matrix", True, 0.1)), (40, 20488, 0, 0, ("rms", "rms", "matrix", True, 0.0)),
                                                    (40, 24584, 0, 0, ("layer", "layer", "none", True, 0.2)), (40, 24584, 0, 0, ("layer", "rms", "vector", True, 0.0)),
                                                    (20, 24583, 1, 1, ("layer", "layer", "matrix", False, 0.1))], ids=str)
def test_gradients_of_clusters_whose_last_block_has_no_columns(ctx, m, n, extra, offset, parts):
    """Nothing of what earlier calls left in shared memory (NaN, here) reaches the others' sums."""
    from paper_2108_08842_b200 import eden

    nan = torch.full((300, 8192), float("nan"), dtype=torch.bfloat16, device="cuda")
    norm = eden.Norm(nan[0], nan[1], "layer")
    ctx.block_join_backward(nan, nan, nan, nan, torch.full((300, 2), float("nan"), device="cuda"), torch.full((300, 2), float("nan"), device="cuda"),
                            after=norm, before=norm, gate=nan)
    T.test_join_backward(ctx, torch.bfloat16, *parts, m, n, extra, offset, False)


@pytest.mark.parametrize("parts", BOTH, ids=lambda p: "-".join(map(str, p)))
def test_exponents_of_a_cluster_at_any_place_of_16_bytes(ctx, parts):
    """Rows of 271 exponents, the second block's 127 of which reach past 128 bytes of their place."""
    T.test_join_backward(ctx, torch.bfloat16, *parts, 150, 8672, 0, 0, True)
