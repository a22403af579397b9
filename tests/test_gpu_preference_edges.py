"""The preference loss where the tests of its formulas do not go: non-finite loss gradients, small probabilities in fp32, long pairs."""
import pytest
import torch

from tests import train_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [33, 1001, 5000, 40000])
@pytest.mark.parametrize("dloss", [float("inf"), float("nan")])
def test_rows_that_are_not_counted_get_zeros_whatever_the_losss_gradient(tr, dtype, vocab, dloss):
    """An infinite or NaN gradient of the loss (an overflowed loss scale) reaches the counted rows only: the others' statistics were never
    written.  Their logits are NaN here, so a row that is read shows."""
    gen = torch.Generator().manual_seed(vocab)
    logits = torch.randn((9, vocab), generator=gen).to(dtype)
    targets = torch.randint(0, vocab, (9,), generator=gen)
    idle = torch.tensor([0, 1, 4, 8])          # two of a prompt, one of another, one outside the sequences
    targets[idle[:3]] = -100
    logits[idle] = float("nan")
    targets[8] = -1
    dev, t = logits.cuda(), targets.cuda()
    out = tr.preference_forward(tr.PreferenceLoss(), dev, t, torch.tensor([0, 4, 8]).cuda())
    out.row_stats[idle.cuda()] = float("nan")  # as uninitialised memory may be
    amax = torch.zeros(1, device="cuda")
    grad = tr.preference_backward(dev, t, out, dloss=torch.tensor([dloss], device="cuda"), amax=amax)
    assert (grad[idle.cuda()] == 0).all()
    assert torch.isnan(grad[2:4]).any() and not torch.isfinite(amax).any()


@pytest.mark.parametrize("rows,vocab,spread", [(6, 1001, 2.0), (40, 32003, 2.0), (4, 50001, 1.0), (300, 517, 12.0), (5, 4099, 30.0)])
def test_fp32_bits(tr, rows, vocab, spread):
    """Every rounding of the fp32 path counted, elements far below the maximum included (bounds in units of 2^-24, d = x - max):
    an exponential   |d| each from the difference and the product, a quarter from log2 e, 4 from the instruction
    a row's sum      its terms' errors by their weight, and as many additions as a term goes through: a thread's share (two halves, 256
                     threads or 32), the halves, 5 + 3 of the joins, a rescaling (4 + 1) at each of the three levels and per new maximum of a
                     thread, of which each adds at most its own share's rounding (4 for the lot)
    logp             the difference |d|, the logarithm 1 + its value, and the last subtraction
    gradient         the quotient 1, an exponential, a product, one addition at the target, for the kernel's own coefficient"""
    gen = torch.Generator().manual_seed(rows + vocab)
    logits = torch.randn((rows, vocab), generator=gen) * spread
    targets = torch.randint(0, vocab, (rows,), generator=gen)
    logits[torch.arange(rows), targets] += 2.0
    cu = torch.tensor([0, rows // 2, rows])
    out = tr.preference_forward(tr.PreferenceLoss(beta=0.3), logits.cuda(), targets.cuda(), cu.cuda())
    grad = tr.preference_backward(logits.cuda(), targets.cuda(), out).cpu().double()
    x = logits.double()
    d = x - x.max(1, keepdim=True).values
    p = torch.softmax(x, 1)
    unit = 2.0 ** -24
    each = 2.25 * d.abs() + 4
    additions = vocab / (2 * 256 if vocab >= 1024 else 2 * 32) + 8 + 1 + 8 + 15 + 4
    total = (p * each).sum(1) + additions                                  # of the row's sum, relative, in units
    at = d[torch.arange(rows), targets]
    lse = torch.logsumexp(d, 1)
    want = at - lse
    assert ((out.logp.cpu().double() - want).abs() <= unit * (at.abs() + total + 1 + 2 * lse.abs() + want.abs())).all()
    one = torch.zeros_like(x)
    one[torch.arange(rows), targets] = 1.0
    c = out.dlogp.cpu().double()[:, None]
    tol = unit * c.abs() * (p * (each + total[:, None] + 3) + one * 2) + 2.0 ** -126       # a product below the normal numbers is flushed
    err = (grad - c * (one - p)).abs()
    assert (err <= tol).all(), float((err / tol).max())
