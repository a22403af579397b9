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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch,rows,cols", [(2, 1, 1), (3, 65, 40), (7, 1024, 64), (5, 24, 3000), (2, 130, 700), (16, 128, 640), (4, 300, 1024), (9, 2000, 8)])
def test_batches(dense, batch, rows, cols, dtype):
    """Each matrix for itself: their sizes differ by 2^40, one is zero, one holds a NaN."""
    g = update((batch, rows, cols), 1)
    g *= torch.exp2(torch.linspace(-20, 20, batch, device="cuda"))[:, None, None]
    g = g.to(dtype)
    g[0] = 0.0
    g[-1, rows // 2, cols // 2] = float("nan")
    got = dense.orthogonalize(g, eps=0.0)
    assert (got[0] == 0).all() and torch.isnan(got[-1]).all()
    if batch > 2:
        assert rel(got[1:-1], orc.orthogonalize(g[1:-1], [orc.QUINTIC] * 5, 0.0)) <= TOL[dtype]
    g[-1, rows // 2, cols // 2] = float("inf")
    assert torch.isnan(dense.orthogonalize(g)[-1]).all()


@pytest.mark.parametrize("rows,cols", [(64, 900), (300, 500), (700, 129)])
@pytest.mark.parametrize("size", [1e-38, 1e30])
def test_sizes_of_values(dense, rows, cols, size):
    g = update((rows, cols), 2, 1.0) * size
    assert rel(dense.orthogonalize(g, eps=0.0), orc.orthogonalize(g, [orc.QUINTIC] * 5, 0.0)) <= TOL[torch.float32]


@pytest.mark.parametrize("rows,cols", [(64, 900), (900, 64), (300, 500), (500, 300)])
def test_coefficients_steps_scale_and_types(dense, rows, cols):
    g = update((rows, cols), 3)
    cubic = [(1.5, -0.5, 0.0)] * 7
    mixed = [(3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0), (1.0, 0.0, 0.0)]
    for table in (cubic, mixed, [(1.0, 0.0, 0.0)], [(0.0, 1.0, 0.0)], [(0.0, 0.0, 1.0)]):
        for scale in (1.0, -0.2):
            assert rel(dense.orthogonalize(g, coefficients=table, scale=scale), orc.orthogonalize(g, table, 1e-7, scale)) <= TOL[torch.float32]
    for steps in (1, 2, 3, 6):
        assert rel(dense.orthogonalize(g, steps=steps), orc.orthogonalize(g, [orc.QUINTIC] * steps, 1e-7)) <= TOL[torch.float32]
    want = orc.orthogonalize(g.bfloat16(), [orc.QUINTIC] * 5, 1e-7)
    assert rel(dense.orthogonalize(g.bfloat16(), dtype=torch.float32), want) <= TOL[torch.float32]
    got = dense.orthogonalize(g, dtype=torch.bfloat16)
    assert got.dtype == torch.bfloat16 and rel(got, orc.orthogonalize(g, [orc.QUINTIC] * 5, 1e-7)) <= TOL[torch.bfloat16]


def test_many_steps(dense):
    """The singular values settle between 0.68 and 1.14, whatever they were: 32 steps of both ways through the library."""
    for rows, cols in ((64, 500), (256, 500)):
        g = update((rows, cols), 4)
        s = torch.linalg.svdvals(dense.orthogonalize(g, steps=32).double())
        assert float(s.min()) > 0.65 and float(s.max()) < 1.2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(64, 400), (401, 63), (300, 257), (512, 512)])
def test_in_place_and_unaligned(dense, rows, cols, dtype):
    g = update((rows, cols), 5).to(dtype)
    want = dense.orthogonalize(g)
    again = g.clone()
    assert torch.equal(dense.orthogonalize(again, out=again), want)
    room = torch.zeros(rows * cols + 8, dtype=dtype, device="cuda")
    odd = room[1:1 + rows * cols].view(rows, cols)
    odd.copy_(g)
    out = torch.full((rows * cols + 8,), 7.0, dtype=dtype, device="cuda")
    got = dense.orthogonalize(odd, out=out[3:3 + rows * cols].view(rows, cols))
    assert rel(got, want.double()) <= 1e-6 if dtype == torch.float32 else torch.equal(got, want)
    assert (out[:3] == 7).all() and (out[3 + rows * cols:] == 7).all()


def test_refusals(dense):
    from paper_2510_24061_b200 import binding as fq
    g = torch.randn((32, 64), device="cuda")
    for bad in (dict(steps=0), dict(steps=33), dict(coefficients=[(1.0, 2.0)]), dict(out=torch.empty((64, 32), device="cuda"))):
        with pytest.raises(ValueError):
            dense.orthogonalize(g, **bad)
    with pytest.raises(ValueError):
        dense.orthogonalize(g.T)
    with pytest.raises(ValueError):
        dense.orthogonalize(g[:0])
    with pytest.raises(TypeError):
        dense.orthogonalize(g.half())
    with pytest.raises(TypeError):
        dense.orthogonalize(g, dtype=torch.float16)
    for table in ([(9.0, 0.0, 0.0)], [(3.0, 0.0, 0.0)] * 3, [(float("nan"), 0.0, 0.0)], [(1.0, 0.0, float("inf"))], [(0.0, 0.0, -8.0)]):
        with pytest.raises(fq.FalqonError):      # values would leave the range that they are held in
            dense.orthogonalize(g, coefficients=table)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(fq.FalqonError):
            dense.orthogonalize(g, eps=eps)
    with pytest.raises(fq.FalqonError):
        dense.orthogonalize(g, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))
