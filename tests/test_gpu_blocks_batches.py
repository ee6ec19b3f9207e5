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
