"""Published schedules of coefficients against the formula in 64 bits, by both ways through the library.

Tolerances, relative to the result's 2-norm.  Five steps of the schedules grow small directions by at most 8.2 * 4.1 * 4 * 3.3 * 2.4 = 1065.  fp32
results: X is held in 22 bits, 2^-23 of its norm, 1.3e-4 after that growth; products tilt its large directions by a few 2^-22 each, without
growth; 1.5e-4.  bf16 results: the first B is up to 8 in size and held in 11
bits, so it leaves up to 8 * 2^-12 / sqrt(3) = 1.1e-3 in X where p(s) is small beside s (0.24 s), which then grows with that direction by at
most 1 / 0.24; and the result's own rounding, 2^-9 / sqrt(3) = 1.1e-3 at most of each value's binade: 1e-2 with the later steps' products."""
import pytest
import torch

from tests import dense_oracle as orc
from tests.test_dense_schedules_host import FIVE, SAFE
from tests.test_gpu_orthogonalize import rel, update

pytestmark = pytest.mark.gpu
TOL = {torch.bfloat16: 1e-2, torch.float32: 1.5e-4}


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def axis(rows, cols):
    """A matrix whose B reaches its bound in single values: one entry with s^2 at the first polynomial's extremum, the rest small."""
    x = torch.full((rows, cols), 1e-4, device="cuda")
    x[3, 5] = 0.826
    x[4, 6] = 0.55
    return x


def axis_bound(g, table, dtype):
    """What held digits leave of `axis` at most, to first order.  Its singular vectors are nearly the axes, so an entry's rounding is its singular
    value's.  Of a value s, with x = s^2, q = b x + c x^2 and p(s) = s (a + q): X's upper part is off by u (relative), G by that twice and its own
    rounding, 3 u, B by |b + 2 c x| x 3 u and its own rounding u |q|, the product B X by u |q| more, so a step leaves (|b + 2 c x| x 3 u + 2 u |q|) / |a + q|
    of p(s), and what the steps before left times |s p'(s) / p(s)|.  u is half a step: 2^-11 of fp16, 2^-22 of two of them.  These
    polynomials cancel (a + q is a fortieth of q) and are steep where they rise again, so five steps in 11 bits leave up to 8 % of such a direction; the
    full schedule, whose last steps are flat at 1, 0.2 %.  To it come the tolerances of other data (the background's directions, the result's rounding)."""
    u = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22
    g = g.double()
    s = torch.linalg.svdvals(g)[:3] / (g.norm() + 1e-7)
    r = torch.zeros_like(s)
    for a, b, c in table:
        x = s * s
        q, slope = b * x + c * x * x, x * (b + 2 * c * x)
        r = (1 + 2 * slope / (a + q)).abs() * r + (3 * u * slope.abs() + 2 * u * q.abs()) / (a + q).abs()
        s = s * (a + q)
    return float((r * s).norm() / s.norm()) + TOL[dtype]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(64, 500), (130, 700), (256, 256), (700, 300), (1024, 1024)])
def test_schedules(dense, rows, cols, dtype):
    for data in (update, axis):
        g = (update((rows, cols)) if data is update else axis(rows, cols)).to(dtype)
        for table in (FIVE, SAFE[:5], SAFE, SAFE + SAFE[-1:] * 4):
            got, want = dense.orthogonalize(g, coefficients=table), orc.orthogonalize(g, table, 1e-7)
            bound = TOL[dtype] if data is update else axis_bound(g, table, dtype)
            assert torch.isfinite(got).all() and rel(got, want) <= bound, (len(table), rel(got, want), bound)


def test_a_schedule_brings_small_singular_values_up(dense):
    """What such schedules are for: singular values from 1.7e-3 to 0.17 of the norm end within 3 % of 1, in eight steps."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    u, _ = torch.linalg.qr(torch.randn((300, 300), generator=gen, device="cuda", dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn((500, 300), generator=gen, device="cuda", dtype=torch.float64))
    s = torch.logspace(-2, 0, 300, device="cuda", dtype=torch.float64)
    g = (u * s) @ v.T
    got = torch.linalg.svdvals(dense.orthogonalize(g.float(), coefficients=SAFE).double())
    assert float(got.min()) > 0.97 and float(got.max()) < 1.03, (float(got.min()), float(got.max()))
