"""8-bit activation checkpoints and the gated MLP that keeps and reads them, against their definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests import train_oracle as orc

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 7), (3, 8), (2, 31), (5, 32), (4, 33), (7, 40), (1, 11008), (33, 1000), (65, 1011), (129, 256), (3, 16384),
          (4500, 1), (3000, 3), (700, 33), (150, 63), (1, 4097), (2, 9001), (1200, 9)]


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


def values(rows, cols, dtype, seed, spread=True):
    """Normal values whose blocks differ in size by many powers of two, with zero blocks and values at the edges of a scale."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=gen)
    if spread:
        x = x * torch.exp2(torch.randint(-12, 12, (rows, cols), generator=gen).float().cummin(1).values)
        if cols >= 64:
            x[0, 32:64] = 0.0
        if cols >= 8:
            x[-1, :8] = torch.tensor([448.0, 449.0, -464.0, 1.75, 0.0, -0.0, 2.0 ** -9, 3.0 * 2.0 ** -10])
    return x.to(dtype)


def check_codes(ck, x):
    e, v = orc.encode(x.double().numpy())
    assert np.array_equal(ck.scales.cpu().numpy(), e)
    got = orc.e4m3_values()[ck.codes.cpu().numpy()]
    assert np.array_equal(got, v, equal_nan=True) and np.array_equal(np.signbit(got[v == 0]), np.signbit(v[v == 0]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_save_and_load_by_definition(tr, rows, cols, dtype):
    x = values(rows, cols, dtype, rows * 131 + cols)
    ck = tr.checkpoint_save(x.cuda())
    check_codes(ck, x)
    want = orc.decode(ck.codes.cpu().numpy(), ck.scales.cpu().numpy())
    for out in (torch.bfloat16, torch.float32):      # every value is 4 significant bits times a power of two: exact in both
        assert np.array_equal(tr.checkpoint_load(ck, out).cpu().double().numpy(), want)


def test_every_code_under_every_scale_reads_back(tr):
    """All 256 x 256 pairs of scale byte and code (a block of 32 codes per scale), against the definition, in fp32; then saving what was
    read gives values that read back the same."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).contiguous()
    scales = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 8).contiguous()
    got = tr.checkpoint_load(tr.Checkpoint(codes.cuda(), scales.cuda()), torch.float32)
    want = orc.decode(codes.numpy(), scales.numpy())
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32)             # 2^127 * 448 is infinite in fp32
    assert np.array_equal(got.cpu().numpy(), want32, equal_nan=True)
    fine = got[:, 1:64]                              # one block and a short one, no NaN codes
    ok = torch.isfinite(fine).all(1)
    again = tr.checkpoint_load(tr.checkpoint_save(fine[ok].contiguous()), torch.float32)
    assert ok.sum() > 240
    big = fine[ok].abs() >= 2.0 ** -126
    assert torch.equal(again[big], fine[ok][big])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [96, 70, 41])
def test_infinities_and_nans_mark_their_block_only(tr, dtype, cols):
    x = values(4, cols, dtype, 5, spread=False)
    x[0, 3], x[1, 33], x[2, cols - 1] = float("inf"), float("nan"), float("-inf")
    ck = tr.checkpoint_save(x.cuda())
    check_codes(ck, x)
    back = tr.checkpoint_load(ck, torch.float32).cpu()
    assert torch.isnan(back[0, :32]).all() and torch.isnan(back[1, 32:min(64, cols)]).all() and torch.isnan(back[2, (cols - 1) // 32 * 32:]).all()
    assert torch.isfinite(back[3]).all() and torch.isfinite(back[1, :32]).all()


def test_the_smallest_and_largest_values(tr):
    """fp32 subnormals (e = 0), and the largest finite value."""
    x = torch.zeros((3, 32))
    x[0] = torch.ldexp(torch.arange(32).float(), torch.tensor(-149))
    x[1] = torch.ldexp(torch.arange(32).float(), torch.tensor(-125))
    x[2, 0], x[2, 1] = torch.finfo(torch.float32).max, -1e38
    ck = tr.checkpoint_save(x.cuda())
    check_codes(ck, x)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_gate_forward(tr, rows, cols, dtype):
    g, u = values(rows, cols, dtype, 1, spread=False) * 3, values(rows, cols, dtype, 2, spread=False)
    amax = torch.zeros(1, device="cuda")
    z, kg, ku = tr.gate_forward(g.cuda(), u.cuda(), amax=amax)
    check_codes(kg, g)
    check_codes(ku, u)
    a, b = g.double(), u.double()
    want = a / (1 + torch.exp(-a)) * b
    # exp, a sum, a quotient and two products in fp32, a few units in the last place each; then the type's rounding
    tol = (orc.type_rounding(dtype) + 2.0 ** -20) * want.abs() + 1e-37
    assert ((z.cpu().double() - want).abs() <= tol).all()
    assert amax.item() == z.float().abs().max().item()
    plain, none, _ = tr.gate_forward(g.cuda(), u.cuda(), save=False)
    assert torch.equal(plain, z) and none is None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_gate_backward(tr, rows, cols, dtype):
    g, u = values(rows, cols, torch.float32, 3, spread=False) * 3, values(rows, cols, torch.float32, 4, spread=False)
    dz = values(rows, cols, dtype, 5, spread=False)
    kg, ku = tr.checkpoint_save(g.cuda()), tr.checkpoint_save(u.cuda())
    ag, au = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    dg, du = tr.gate_backward(kg, ku, dz.cuda(), amax_dg=ag, amax_du=au)
    a, b = (torch.from_numpy(orc.decode(k.codes.cpu().numpy(), k.scales.cpu().numpy())) for k in (kg, ku))
    t = dz.double()
    s = torch.sigmoid(a)
    for got, want, size in ((dg, t * b * s * (1 + a * (1 - s)), (t * b * s).abs() * (1 + a.abs() * (1 - s))), (du, t * a * s, (t * a * s).abs())):
        tol = orc.type_rounding(dtype) * want.abs() + 2.0 ** -19 * size + 1e-37
        assert ((got.cpu().double() - want).abs() <= tol).all()
    assert ag.item() == dg.float().abs().max().item() and au.item() == du.float().abs().max().item()
    # in place, and against differences of the forward in 64 bits
    again = dz.cuda()
    dg2, du2 = tr.gate_backward(kg, ku, again, dg=again)
    assert torch.equal(dg2, dg) and torch.equal(du2, du) and dg2.data_ptr() == again.data_ptr()
    h = 1e-5
    f = lambda a, b: a / (1 + torch.exp(-a)) * b  # noqa: E731
    diff = t * (f(a + h, b) - f(a - h, b)) / (2 * h)
    assert ((dg.cpu().double() - diff).abs() <= (2 * orc.type_rounding(dtype) + 1e-6) * (t.abs() * (1 + a.abs()) * (1 + b.abs()))).all()


def test_offsets_beyond_32_bits(tr):
    """A tensor of more than 2^31 values: the last row is where a 32-bit offset would wrap."""
    rows, cols = 131080, 16384                       # 2.15e9 values: 4.3 GB in bf16
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.linspace(-3, 3, cols).to(torch.bfloat16)
    ck = tr.checkpoint_save(x)
    last = x[-1:].cpu()
    check_codes(tr.Checkpoint(ck.codes[-1:], ck.scales[-1:]), last)
    assert int(ck.codes[:-1].max()) == 0
    del x
    back = tr.checkpoint_load(ck)
    want = orc.decode(ck.codes[-1:].cpu().numpy(), ck.scales[-1:].cpu().numpy())
    assert np.array_equal(back[-1:].cpu().double().numpy(), want)
