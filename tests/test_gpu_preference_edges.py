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
