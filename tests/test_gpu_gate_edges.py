"""The gated MLP where exp(-g) is huge or tiny, with bounds that follow from the arithmetic instead of an absolute allowance."""
import numpy as np
import pytest
import torch

from tests import train_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


def gates(cols, dtype):
    """Every order of size on both sides: -104 .. 104, dense where the sigmoid leaves the normal numbers (-87.34 on)."""
    x = torch.cat([torch.linspace(-104.0, 104.0, 3001), torch.linspace(-92.5, -86.5, 997), torch.tensor([0.0, -0.0, -3.0e38, 3.0e38])])
    rows = -(-x.numel() // cols)
    return torch.cat([x, torch.zeros(rows * cols - x.numel())]).view(rows, cols).to(dtype)


# A sigmoid's relative error: fp32 expf and three roundings (2 + 3 halves of 2^-23), bf16 a rounded exponent (|g| * 2^-24 and that much again
# from log2 e's own rounding) and two instructions of 2 * 2^-23; plus a subnormal one's spacing, half of 2^-149 each of exp and product.
def sigmoid_error(g, s, dtype):
    rel = 4 * 2.0 ** -23 if dtype == torch.float32 else g.abs() * 2.0 ** -23 + 8 * 2.0 ** -23
    return rel * s + 2.0 ** -149


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [64, 40, 41])
def test_forward_down_to_the_smallest_normal_results(tr, dtype, cols):
    g = gates(cols, dtype)
    u = torch.where(torch.arange(g.numel()).view(g.shape) % 3 == 0, 1.0, -3.0).to(dtype)
    z, _, _ = tr.gate_forward(g.cuda(), u.cuda())
    a, b = g.double(), u.double()
    s = torch.sigmoid(a)
    want = a * s * b
    # the sigmoid, two products (2^-24 each), the type's rounding; where the result is subnormal in its type, that spacing (2^-133 for bf16)
    tol = (a * b).abs() * sigmoid_error(a, s, dtype) + (orc.type_rounding(dtype) + 2 * 2.0 ** -24) * want.abs() + (2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -148)
    over = want.abs() > torch.finfo(dtype).max       # 3e38 times 3: infinite when rounded to the type
    assert torch.equal(z.cpu().double()[over], want[over].to(dtype).double()) and over.any() and over.sum() < 3
    err = torch.where(over, 0.0, (z.cpu().double() - want).abs())
    assert (err <= tol).all(), (float((err / tol).max()), float(g.flatten()[(err / tol).argmax()]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [64, 40, 41])
def test_backward_down_to_the_smallest_normal_results(tr, dtype, cols):
    g = gates(cols, torch.float32)
    g[g.abs() > 1e30] = 0.0                         # a block's scale is that of its largest value: these have a row of their own below
    # a value to a block, so that its scale is its own: the code keeps four significant bits of each
    wide = torch.zeros((g.numel(), cols))
    wide[:, 0] = g.flatten()
    kg = tr.checkpoint_save(wide.cuda())
    ku = tr.checkpoint_save(torch.full_like(wide, -1.5).cuda())
    dz = torch.full_like(wide, 0.75).to(dtype)
    dg, du = tr.gate_backward(kg, ku, dz.cuda())
    a = torch.from_numpy(orc.decode(kg.codes.cpu().numpy(), kg.scales.cpu().numpy()))
    b = torch.from_numpy(orc.decode(ku.codes.cpu().numpy(), ku.scales.cpu().numpy()))
    t, s = dz.double(), torch.sigmoid(a)
    e = sigmoid_error(a, s, dtype)
    low = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -148
    # du: the sigmoid and two products; dg = dz u (s + g s (1 - s)): the sigmoid enters three times, 1 - s is off by 2^-24 besides
    want = t * a * s
    assert ((du.cpu().double() - want).abs() <= (t * a).abs() * e + (orc.type_rounding(dtype) + 2 * 2.0 ** -24) * want.abs() + low).all()
    want = t * b * (s + a * s * (1 - s))
    size = (t * b).abs() * (e * (1 + 2 * a.abs()) + 6 * 2.0 ** -24 * s * (1 + a.abs()))
    err = (dg.cpu().double() - want).abs()
    tol = size + orc.type_rounding(dtype) * want.abs() + low
    assert (err <= tol).all(), float((err / tol).max())


def test_infinite_gates(tr):
    """silu(inf) = inf; silu(-inf) = -inf * 0 is NaN, as in the formula; both only in their place, and their blocks read back as NaN."""
    for dtype in (torch.bfloat16, torch.float32):
        g = torch.ones((2, 96), dtype=dtype)
        g[0, 3], g[1, 40] = float("inf"), float("-inf")
        z, kg, _ = tr.gate_forward(g.cuda(), torch.ones_like(g).cuda())
        assert torch.isinf(z[0, 3]) and z[0, 3] > 0 and torch.isnan(z[1, 40])
        z[0, 3] = z[1, 40] = 0.0
        assert torch.isfinite(z).all()
        back = tr.checkpoint_load(kg, torch.float32).cpu()
        assert torch.isnan(back[0, :32]).all() and torch.isnan(back[1, 32:64]).all() and torch.isfinite(back[0, 32:]).all()
        assert np.array_equal(kg.scales.cpu().numpy() == 255, np.array([[1, 0, 0], [0, 1, 0]], dtype=bool))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(300, 1024), (33, 1000), (65, 1011), (1, 7), (700, 33)])
def test_backward_with_either_gradient_in_place(tr, rows, cols, dtype):
    gen = torch.Generator().manual_seed(cols)
    kg, ku = (tr.checkpoint_save(torch.randn((rows, cols), generator=gen).cuda()) for _ in range(2))
    dz = torch.randn((rows, cols), generator=gen).to(dtype).cuda()
    want = tr.gate_backward(kg, ku, dz)
    for which in ("dg", "du"):
        into = dz.clone()
        got = tr.gate_backward(kg, ku, into, **{which: into})
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[which == "du"].data_ptr() == into.data_ptr()
