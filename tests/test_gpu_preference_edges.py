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


def pairs_from(logp, targets, cu, ref, spec):
    """seq_logp, pair_loss and dlogp in 64 bits from the rows' log-probabilities as the call returned them."""
    f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    beta, margin, eps, weight = f(spec.beta), f(spec.margin), f(spec.label_smoothing), f(spec.nll_weight)
    counted, n, total = targets >= 0, [], []
    for a, b in zip(cu, cu[1:]):
        n.append(max(int(counted[a:b].sum()), 1))
        total.append(logp[a:b].sum())
    total, n = torch.stack(total), torch.tensor(n, dtype=torch.float64)
    seq = total / n if spec.average else total
    u = (seq - ref)[0::2] - (seq - ref)[1::2]
    D = beta * u - margin
    sp = torch.nn.functional.softplus
    if spec.kind == "sigmoid":
        # softplus in torch returns D itself beyond a threshold of 20, so its second term is added
        tail = torch.log1p(torch.exp(-D.abs()))
        l = (1 - eps) * (torch.relu(-D) + tail) + eps * (torch.relu(D) + tail)
        du = beta * (eps * torch.sigmoid(D) - (1 - eps) * torch.sigmoid(-D))
    elif spec.kind == "hinge":
        l, du = torch.relu(1 - D), torch.where(D < 1, -beta, torch.where(D >= 1, 0.0, D))      # the slope of a NaN is one
    else:
        l, du = (u - margin - 0.5 / beta) ** 2, 2 * (u - margin - 0.5 / beta)
    nll = weight / n[0::2]
    coef = torch.stack(((du / n[0::2] if spec.average else du) - nll, -(du / n[1::2] if spec.average else du)), 1).view(-1) / len(u)
    dlogp = torch.zeros_like(logp)
    for i, (a, b) in enumerate(zip(cu, cu[1:])):
        dlogp[a:b] = torch.where(counted[a:b], coef[i], 0.0)
    return seq, l - nll * total[0::2] if weight else l.clone(), dlogp, l, (du.abs() + (nll if spec.average else nll)), D


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.1), ("hinge", 0.0), ("ipo", 0.0)])
def test_the_pairs_arithmetic_is_rounded_once(tr, kind, smoothing, average):
    """From the returned logp on: sums, differences and results are 64 bits and rounded once (2^-24); the sigmoid's exponential, logarithm and
    reciprocal are 32 bits and enter with 4 * 2^-23 of their own values.  References lie close to the policy's own sums, as early in training,
    so that u is small beside them; margins bring the loss near its bends."""
    lens = [int(v) for v in torch.randint(1, 60, (64,), generator=torch.Generator().manual_seed(3))]
    cu = torch.tensor([0] + lens).cumsum(0)
    rows, vocab = int(cu[-1]), 200
    gen = torch.Generator().manual_seed(4)
    logits = torch.randn((rows, vocab), generator=gen) * 2
    targets = torch.randint(0, vocab, (rows,), generator=gen)
    targets[torch.rand(rows, generator=gen) < 0.25] = -100
    first, _ = tr.sequence_logprob(logits.cuda(), targets.cuda(), cu.cuda(), average=average)
    ref = (first.cpu() + torch.randn(64, generator=gen) * 0.05).contiguous()
    for beta, margin, nll in ((0.1, 0.0, 0.0), (2.0, 0.9, 0.0), (30.0, 0.0, 0.3), (0.5, -12.0, 0.0), (0.5, 60.0, 0.0)):
        spec = tr.PreferenceLoss(kind, beta, margin, smoothing, average, nll)
        out = tr.preference_forward(spec, logits.cuda(), targets.cuda(), cu.cuda(), ref.cuda())
        seq, loss, dlogp, l, size, D = pairs_from(out.logp.cpu().double(), targets, cu.tolist(), ref.double(), spec)
        soft = (4 * 2.0 ** -23 if kind == "sigmoid" else 0.0)
        once = 2.0 ** -24 * (1 + 2.0 ** -20)
        assert ((out.seq_logp.cpu().double() - seq).abs() <= once * seq.abs() + 2.0 ** -149).all()
        err, tol = (out.pair_loss.cpu().double() - loss).abs(), once * loss.abs() + soft * l.abs() + 2.0 ** -126 + 2.0 ** -48 * seq.abs().max()
        assert (err <= tol).all(), (beta, margin, float((err / tol).max()))
        per = (size / len(size)).repeat_interleave(2)
        bound = torch.cat([per[i].expand(b - a) for i, (a, b) in enumerate(zip(cu.tolist(), cu.tolist()[1:]))])
        err, tol = (out.dlogp.cpu().double() - dlogp).abs(), once * dlogp.abs() + soft * bound + 2.0 ** -126 + 2.0 ** -48 * seq.abs().max()
        assert (err <= tol).all(), (beta, margin, float((err / tol).max()))
        assert abs(out.loss.item() - float(loss.mean())) <= 2.0 ** -23 * float(loss.abs().mean()) + soft * float(l.mean()) + 2.0 ** -48 * float(seq.abs().max())


def check_skewed(tr, lens, vocab, seed, average, threads=None):
    """logp, seq_logp, dlogp and the gradient where sequences differ much in length, rows counted and not in turn."""
    cu = torch.tensor([0] + lens).cumsum(0)
    rows, gen = sum(lens), torch.Generator().manual_seed(seed)
    logits = torch.randn((rows, vocab), generator=gen) * 2
    targets = torch.randint(0, vocab, (rows,), generator=gen)
    targets[torch.rand(rows, generator=gen) < 0.4] = -100
    spec = tr.PreferenceLoss("sigmoid", 0.01, 0.0, 0.1, average, 0.2)
    call = lambda: tr.preference_forward(spec, logits.cuda(), targets.cuda(), cu.cuda())  # noqa: E731
    out = call()
    if threads is not None:
        from tests.launches import launched
        dev = logits.cuda(), targets.cuda(), cu.cuda()
        (used,) = [t for n, _, t in launched(lambda: tr.preference_forward(spec, *dev)) if "sequence_kernel" in n]
        assert used == threads
    ref = torch.zeros(len(lens), dtype=torch.float64)
    logp = torch.where(targets >= 0, torch.log_softmax(logits.double(), 1)[torch.arange(rows), targets.clamp(min=0)], 0.0)
    assert float((out.logp.cpu().double() - logp).abs().max()) <= 2.0 ** -18                # a few units of 2^-23 of |d| + lse, below 20
    seq, loss, dlogp, l, size, _ = pairs_from(out.logp.cpu().double(), targets, cu.tolist(), ref, spec)
    soft, once = 4 * 2.0 ** -23, 2.0 ** -24 * (1 + 2.0 ** -20)
    assert ((out.seq_logp.cpu().double() - seq).abs() <= once * seq.abs() + 2.0 ** -149).all()
    assert ((out.pair_loss.cpu().double() - loss).abs() <= once * loss.abs() + soft * l.abs() + 2.0 ** -40).all()
    got = out.dlogp.cpu().double()
    assert ((got == 0) == (targets < 0)).all()
    per = (size / len(size)).repeat_interleave(2).repeat_interleave(torch.tensor(lens))
    assert ((got - dlogp).abs() <= once * dlogp.abs() + soft * per + 2.0 ** -126).all()
    grad = tr.preference_backward(logits.cuda(), targets.cuda(), out).cpu().double()
    one = torch.zeros((rows, vocab), dtype=torch.float64)
    one[torch.arange(rows), targets.clamp(min=0)] = 1.0
    want = got[:, None] * (one - torch.softmax(logits.double(), 1))
    assert ((grad - want).abs() <= 2.0 ** -18 * got.abs()[:, None]).all()


@pytest.mark.parametrize("average", [False, True])
def test_many_short_pairs_and_one_long(tr, average):
    """The CTA of a pair is sized by the average: it has to stay able to walk a long one."""
    check_skewed(tr, [1, 1] * 699 + [2300, 2100], 40, 5, average, threads=128)
    check_skewed(tr, [1, 0, 700, 3] + [2, 1] * 40, 2100, 6, average, threads=128)


@pytest.mark.parametrize("average", [False, True])
def test_more_rows_than_a_thread_remembers(tr, average):
    """A thread keeps the marks of its first 64 rows and reads the others' again: 64 * 128 rows and more in one pair of many, and 64 * 1024 in
    the only pair."""
    check_skewed(tr, [1, 1] * 500 + [5000, 4500], 12, 7, average, threads=128)
    check_skewed(tr, [36000, 35001], 7, 8, average, threads=1024)


@pytest.mark.parametrize("dtype,k", [(torch.bfloat16, 1), (torch.float32, 2)])
@pytest.mark.parametrize("rows,vocab,warps", [(300, 2000, False), (300, 1000, True), (1000, 3990, True), (1000, 4100, False), (3990, 6000, False), (4000, 8100, True),
                                              (4000, 8200, False), (12000, 2500, True), (49, 1000, False), (2, 6, True)])
def test_a_warp_or_a_cta_to_a_row(tr, rows, vocab, warps, dtype, k):
    """Both passes by the same rule, which looks at rows and columns."""
    from tests.launches import launched
    logits = torch.zeros((rows, vocab // k), dtype=dtype, device="cuda")
    targets, cu = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.tensor([0, rows // 2, rows], device="cuda")
    def call():
        out = tr.preference_forward(tr.PreferenceLoss(), logits, targets, cu)
        return tr.preference_backward(logits, targets, out), out
    used = {n: c for n, c, _ in launched(call) if "row_stats" in n or "logit_grad" in n}
    assert len(used) == 2
    for name, ctas in used.items():
        assert ("Li32E" in name) == warps and (ctas == -(-rows // 8)) == warps, name


@pytest.mark.parametrize("rows,vocab", [(1000, 2040), (4100, 2051), (4000, 4090)])
def test_longer_rows_by_warps(tr, rows, vocab):
    check_skewed(tr, [rows // 3, rows - rows // 3], vocab, vocab, False)


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.1), ("hinge", 0.0), ("ipo", 0.0)])
def test_targets_that_cannot_be(tr, kind, smoothing, average):
    """A target whose logit is -inf in the chosen, the rejected, both or neither sequence: infinite log-probabilities go through the pair's
    arithmetic as through the formulas, and the other pairs are as without them."""
    cu = torch.arange(0, 17, 2)
    logits = torch.randn((16, 50), generator=torch.Generator().manual_seed(11))
    targets = torch.arange(16) % 50
    for row in (1, 6, 8, 10):                    # pair 0: chosen; pair 1: rejected; pair 2: both; pair 3: neither
        logits[row, targets[row]] = float("-inf")
    for nll in (0.0, 0.5):
        spec = tr.PreferenceLoss(kind, 0.5, 0.25, smoothing, average, nll)
        out = tr.preference_forward(spec, logits.cuda(), targets.cuda(), cu.cuda())
        logp = out.logp.cpu().double()
        assert torch.equal(torch.isinf(logp), torch.isin(torch.arange(16), torch.tensor([1, 6, 8, 10])))
        seq, loss, dlogp, _, _, D = pairs_from(logp, targets, cu.tolist(), torch.zeros(8, dtype=torch.float64), spec)
        if kind == "sigmoid" and smoothing == 0.0:
            loss[1] = 0.0 + (-0.0 if nll == 0.0 else -nll / 2 * float(logp[4:6].sum()))     # 0 * inf of the other term is left out
        assert torch.isinf(D[0]) and D[0] < 0 and torch.isinf(D[1]) and D[1] > 0 and torch.isnan(D[2]) and torch.isfinite(D[3])
        for got, want in ((out.seq_logp, seq), (out.pair_loss, loss), (out.dlogp, dlogp)):
            assert torch.allclose(got.cpu().double(), want, rtol=2.0 ** -21, atol=2.0 ** -30, equal_nan=True), (got, want)
        assert torch.isnan(out.loss)
