"""The result's scale over fp32's range, by both ways through the library.  Tolerances as for a scale of 1: the last multiplication is off by half a step,
and results are normal numbers of their type here but for single values far below the others."""
import pytest
import torch

from tests import dense_oracle as orc
from tests.test_gpu_orthogonalize import TOL, rel, update

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(64, 500), (300, 500), (500, 301)])
@pytest.mark.parametrize("scale", [0.0, 3e-34, -7e-32, 1e-20, 0.3, 3e38])
def test_scale(dense, rows, cols, dtype, scale):
    g = update((rows, cols), 21).to(dtype)
    got, want = dense.orthogonalize(g, scale=scale), orc.orthogonalize(g, [orc.QUINTIC] * 5, 1e-7, scale)
    if scale == 0.0:
        assert not got.any()
    else:
        assert torch.isfinite(got).all() and rel(got, want) <= TOL[dtype], rel(got, want)


@pytest.mark.parametrize("rows,cols", [(64, 500), (300, 500)])
def test_a_scale_that_undoes_a_large_eps(dense, rows, cols):
    """|g| is 1e-30 of eps: the result would leave fp32's range but for the scale."""
    g = update((rows, cols), 22)
    g = g / g.norm()
    got, want = dense.orthogonalize(g, eps=1e38, scale=1e38), orc.orthogonalize(g, [orc.QUINTIC] * 5, 1e38, 1e38)
    assert rel(got, want) <= TOL[torch.float32], rel(got, want)
