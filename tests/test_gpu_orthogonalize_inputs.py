"""Orthogonalised updates of what the other tests do not draw: gradients of low rank with little or no noise, as adapters' are, and many steps by
way of the Gram matrix.  Against the formula in 64 bits, relative to the result's 2-norm.

Low rank.  X is held in 22 bits: what that leaves, at most 2^-23 of its norm, lies in all directions, those without anything in them too, and
grows there by 3.4445 a step: 2^-23 * 3.4445^5 = 5.8e-5 of the first X and, with what is left by the later ones, 1 / (1 - 1 / 3.4445) times as
much, of a result whose norm is 0.68 at least: 1.2e-4.  (Products tilt the large directions, by a few 2^-22 a step, which does not grow.)  Plain
fp32 products leave more of it.  bf16 results as for other data: X is held as well, products tilt by some 2^-12 a step.
Many steps: results by the Gram matrix in fp64 carry their own rounding and at most 2^-24 (the rule that admits them): 2e-7."""
import pytest
import torch

from tests import dense_oracle as orc
from tests.launches import launched
from tests.test_gpu_orthogonalize import rel, update

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def low_rank(rows, cols, rank, noise):
    g = torch.Generator(device="cuda").manual_seed(rows + rank)
    x = torch.randn((rows, rank), generator=g, device="cuda") @ torch.randn((rank, cols), generator=g, device="cuda")
    return x + noise * torch.randn((rows, cols), generator=g, device="cuda")


@pytest.mark.parametrize("rows,cols", [(130, 700), (256, 256), (1000, 300), (1024, 1024), (130, 4096), (64, 900)])
@pytest.mark.parametrize("rank,noise", [(1, 0.0), (1, 1e-6), (1, 1e-3), (4, 0.0), (4, 1e-3), (16, 1e-4)])
def test_low_rank(dense, rows, cols, rank, noise):
    g = low_rank(rows, cols, rank, noise)
    assert rel(dense.orthogonalize(g), orc.orthogonalize(g, [orc.QUINTIC] * 5, 1e-7)) <= 1.2e-4
    h = g.bfloat16()
    assert rel(dense.orthogonalize(h), orc.orthogonalize(h, [orc.QUINTIC] * 5, 1e-7)) <= 5e-3


@pytest.mark.parametrize("rows,cols", [(64, 500), (500, 30), (128, 500), (900, 100)])       # two buffers, and one
@pytest.mark.parametrize("table", [[(1.5, -0.5, 0.0)] * 20, [(1.5, -0.5, 0.0)] * 23, [(1.0, -0.2, 0.05)] * 32, [(1.5, -0.5, 0.0), (1.0, 0.0, 0.0)] * 16])
def test_many_steps_by_the_gram_matrix(dense, rows, cols, table):
    g = update((3, rows, cols), 6)
    ran = [k for k, *_ in launched(lambda: dense.orthogonalize(g, coefficients=table))]
    assert len(ran) == 3 and "thin_gram" in ran[0], ran
    got, want = dense.orthogonalize(g, coefficients=table), orc.orthogonalize(g, table, 1e-7)
    assert rel(got, want) <= 2e-7, rel(got, want)


@pytest.mark.parametrize("rows,cols", [(65, 700), (69, 759), (3955, 69), (75, 381), (96, 2000), (90, 91), (97, 3000), (300, 700)])
def test_bf16_results_beside_their_own_rounding(dense, rows, cols):
    """A strong part of rank 32 and noise, as an optimizer's momentum: no more than 1.5 times what rounding the exact results to bf16 leaves.  What is held
    in 11 bits is off by 2^-11 / sqrt(12) * 1.4 of itself on average (1.9e-4), and a step takes G (which is then exact for B), B and X so.  For short sides up to
    96 only G's rounding is left, 1.1 to 1.15 times by the products' model; for longer ones all three, averaged over the short side, up to 1.45 times at 97."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    k = min(rows, cols, 32)
    x = torch.randn((rows, k), generator=g, device="cuda") / torch.arange(1, k + 1, device="cuda") @ torch.randn((k, cols), generator=g, device="cuda")
    x = ((x + 0.5 * torch.randn((rows, cols), generator=g, device="cuda")) * 1e-3).bfloat16()
    want = orc.orthogonalize(x, [orc.QUINTIC] * 5, 1e-7)
    least = rel(want.bfloat16(), want)
    assert rel(dense.orthogonalize(x), want) <= 1.5 * least, rel(dense.orthogonalize(x), want) / least


@pytest.mark.parametrize("rows,cols", [(129, 977), (143, 977), (9953, 146), (530, 147), (403, 6139), (133, 232), (300, 700), (1106, 388)])
def test_fp32_results_beside_plain_products(dense, rows, cols):
    """As exact as plain fp32 products of the same steps, but for half as much again (sums that are cut off instead of rounded): the same inputs, whose
    singular values come together after four steps, where the fifth multiplies what is systematic in them."""
    assert not torch.backends.cuda.matmul.allow_tf32
    g = torch.Generator(device="cuda").manual_seed(cols)
    k = min(rows, cols, 32)
    g = (torch.randn((rows, k), generator=g, device="cuda") / torch.arange(1, k + 1, device="cuda") @ torch.randn((k, cols), generator=g, device="cuda")
         + 0.5 * torch.randn((rows, cols), generator=g, device="cuda")) * 1e-3
    want = orc.orthogonalize(g, [orc.QUINTIC] * 5, 1e-7)
    x = g.mT if rows > cols else g
    x = x / (x.double().norm() + 1e-7).float()
    a, b, c = orc.QUINTIC
    for _ in range(5):
        m = x @ x.mT
        x = a * x + (b * m + c * (m @ m)) @ x
    plain, got = rel(x.mT if rows > cols else x, want), rel(dense.orthogonalize(g), want)
    assert got <= 1.5 * plain, (got, plain)
