"""Orthogonalised updates at the ends of their range: norms far below eps.  Against the formula in 64 bits.

Tolerances as for ordinary norms (test_gpu_orthogonalize.py), relative to the result's 2-norm: where |g| is far below eps the formula only
multiplies X, by its first coefficient a step, and what is held is held in as many digits."""
import pytest
import torch

from tests import dense_oracle as orc
from tests.test_gpu_orthogonalize import TOL, rel, update

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def of_norm(g, norm):
    return g * (norm / g.flatten(-2).norm(dim=-1))[..., None, None]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(64, 500), (130, 700), (300, 500), (500, 300), (1024, 1024), (257, 2048)])
@pytest.mark.parametrize("below", [0.3, 1e-2, 1e-4, 1e-6, 1e-7, 1e-12])
def test_norms_below_eps(dense, rows, cols, dtype, below):
    g = of_norm(update((rows, cols), 11), 1e-7 * below).to(dtype)
    for steps in (1, 5, 9):
        got, want = dense.orthogonalize(g, steps=steps), orc.orthogonalize(g, [orc.QUINTIC] * steps, 1e-7)
        assert rel(got, want) <= TOL[dtype], (steps, rel(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(70, 900), (700, 300), (200, 200)])
def test_a_batch_on_both_sides_of_eps(dense, rows, cols, dtype):
    """Each matrix has its own exponent: norms from 2^-70 to 2^20 of eps, a zero, a NaN."""
    norms = torch.exp2(torch.tensor([-70.0, -45.0, -20.0, -8.0, -3.0, -1.0, 0.0, 1.0, 20.0], device="cuda", dtype=torch.float64)) * 1e-7
    g = of_norm(update((11, rows, cols), 12).double(), torch.cat([norms, norms[:2]])).to(dtype)
    g[-2], g[-1, 3, 5] = 0.0, float("nan")
    tables = [[orc.QUINTIC] * 5, [(1.5, -0.5, 0.0)] * 6, [(0.5, 0.25, 0.0)] * 3, [(2.0, -1.5, 0.5), (0.0, 1.0, 0.0), (1.5, -0.5, 0.0)]]
    for table in tables[:3] if dtype == torch.bfloat16 else tables:
        got = dense.orthogonalize(g, coefficients=table, scale=-0.2)
        assert (got[-2] == 0).all() and torch.isnan(got[-1]).all()
        want = orc.orthogonalize(g[:-2], table, 1e-7, -0.2)
        seen = want.flatten(-2).norm(dim=-1) > 1e-30       # (s^3 of the smallest leaves fp32's range)
        assert rel(got[:-2][seen], want[seen]) <= TOL[dtype], (table[0], rel(got[:-2][seen], want[seen]))


@pytest.mark.parametrize("rows,cols", [(300, 500), (500, 300)])
def test_a_large_eps(dense, rows, cols):
    """eps is a float like any other: norms of 1 under an eps of 1e20 and of 1e30."""
    g = of_norm(update((rows, cols), 13), 1.0)
    for eps in (1e20, 1e30):
        assert rel(dense.orthogonalize(g, eps=eps), orc.orthogonalize(g, [orc.QUINTIC] * 5, eps)) <= TOL[torch.float32]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(300, 700), (700, 130)])
def test_captured_on_both_sides_of_eps(dense, rows, cols, dtype):
    """A captured call finds each input's own exponents, in place too, and gives what an eager call gives."""
    g = of_norm(update((3, rows, cols), 14), 1.0).to(dtype)
    held = g.clone()
    dense.orthogonalize(held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dense.orthogonalize(held, out=held)
    for sizes in ((1.0, 1e-9, 1e-12), (1e-14, 1.0, 1e-7), (1.0, 1.0, 1.0)):
        x = (g.double() * torch.tensor(sizes, device="cuda", dtype=torch.float64)[:, None, None]).to(dtype)
        held.copy_(x)
        graph.replay()
        assert torch.equal(held, dense.orthogonalize(x))
        assert rel(held, orc.orthogonalize(x, [orc.QUINTIC] * 5, 1e-7)) <= TOL[dtype]
