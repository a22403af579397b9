"""Updates orthogonalised by Newton-Schulz products, against the formula in 64 bits.

Tolerances, relative to the result's 2-norm.  bf16 results: their own rounding, at most 2^-9 of each value, and the products of fp16 operands
(2^-12 of each value of G, B and X, random in sign): of a step's three products each leaves sqrt(3) * 2^-12 at most, later steps
multiply by at most |d(p(s))/ds| = 3.45 in directions that still grow, which in size are small beside those that have; so 2^-9 and a few 2^-12:
5e-3.  fp32 results: 22-bit operands and fp32 sums, which plain fp32 products have as well: a step's three products are off by a few
2^-22 each, five steps of growth by at most 3.45^5 = 490 in directions that are small, 1e-5 (what plain fp32 products leave is 1e-6 to 5e-6)."""
import pytest
import torch

from tests import dense_oracle as orc

pytestmark = pytest.mark.gpu
TOL = {torch.bfloat16: 5e-3, torch.float32: 1e-5}


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def update(shape, seed=0, size=1e-3, rank=16):
    """A gradient as the optimizer sees it: a strong part of low rank, and noise."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    *b, rows, cols = shape
    k = min(rows, cols, rank)
    fall = 1.0 / torch.arange(1, k + 1, device="cuda")
    x = torch.randn((*b, rows, k), generator=g, device="cuda") * fall @ torch.randn((*b, k, cols), generator=g, device="cuda")
    return (x + 0.5 * torch.randn(shape, generator=g, device="cuda")) * size


def rel(got, want):
    d = (got.double() - want).flatten(-2).norm(dim=-1) / want.flatten(-2).norm(dim=-1)
    return float(d.max())


SHAPES = [(1, 1), (1, 100), (100, 1), (3, 7), (16, 16), (64, 64), (63, 129), (129, 63), (128, 1000), (1000, 128), (200, 4096), (256, 256), (257, 300),
          (500, 333), (512, 1024), (1024, 512), (777, 1531), (1300, 1100), (64, 8192), (8192, 64)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_against_64_bits(dense, rows, cols, dtype):
    g = update((rows, cols)).to(dtype)
    want = orc.orthogonalize(g, [orc.QUINTIC] * 5, 1e-7)
    got = dense.orthogonalize(g)
    assert got.dtype == dtype and rel(got, want) <= TOL[dtype], rel(got, want)
