"""The preference loss of paired sequences and the sequence log-probabilities, against 64 bits."""
import pytest
import torch

from tests import train_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


@pytest.fixture(scope="module")
def fq():
    from paper_2510_24061_b200 import binding
    return binding


def make(rows, vocab, cu, dtype, seed, pitch=None, offset=0, scale=2.0):
    """Logits in a buffer of the given row pitch that starts `offset` values after a 16-byte boundary, filled with NaN around them."""
    gen = torch.Generator().manual_seed(seed)
    pitch = vocab if pitch is None else pitch
    store = torch.full((offset + rows * pitch + 8,), float("nan"), dtype=dtype)
    logits = store[offset:offset + rows * pitch].view(rows, pitch)[:, :vocab]
    logits.copy_(torch.randn((rows, vocab), generator=gen) * scale)
    targets = torch.randint(0, vocab, (rows,), generator=gen)
    logits[torch.arange(rows), targets] += 4.0
    for a, b in zip(cu, cu[1:]):
        targets[a:a + (b - a) // 3] = -100
    ref = torch.randn(len(cu) - 1, generator=gen)
    dev = store.cuda()[offset:offset + rows * pitch].view(rows, pitch)[:, :vocab]
    return logits, dev, targets, torch.tensor(cu, dtype=torch.int64), ref


# rows, vocab, sequence bounds, row pitch beyond the vocabulary, offset of the first value: one row to several parts per row; odd
# vocabularies, shorter than a vector, rows that start anywhere; sequences of length zero, single tokens, rows outside
CASES = [
    (2, 1, [0, 1, 2], 0, 0), (2, 5, [0, 1, 2], 0, 0), (7, 3, [0, 0, 3, 5, 7], 0, 1), (9, 33, [0, 4, 9], 0, 0), (24, 1000, [0, 6, 12, 18, 24], 0, 0),
    (13, 1001, [0, 6, 13], 3, 1), (6, 4099, [0, 3, 6], 0, 3), (3, 32000, [0, 1, 3], 0, 0), (40, 32003, [0, 11, 20, 33, 40], 0, 0),
    (5, 50001, [0, 2, 5], 7, 5), (600, 2048, [0, 100, 350, 351, 600], 0, 0), (1300, 517, [0, 650, 1300], 0, 0), (4, 131072, [0, 2, 4], 0, 0),
]
LOSSES = [("sigmoid", 0.0, False, 0.0), ("sigmoid", 0.1, True, 0.3), ("hinge", 0.0, False, 0.0), ("ipo", 0.0, True, 0.0)]


def bounds(ref, kind, beta, logits, average):
    """Error of a row's log-probability: the sum of exponentials (a unit in the 22nd bit each and up to 2^8 additions in a thread's
    share and its joins: 2^-15 of it at worst, as a difference of its logarithm), the logarithm, the difference; and what follows."""
    row = 2.0 ** -15 + 2.0 ** -22 * logits.double().abs().max()
    n = 1.0 if average else float(ref["counted"].sum())
    u = 2 * row * n
    slope = {"sigmoid": beta, "hinge": beta, "ipo": float(2 * ref["u"].abs().max() + 1 / beta)}[kind]
    curve = {"sigmoid": beta * beta / 4, "hinge": 0.0, "ipo": 2.0}[kind]
    return row, u, slope, curve


@pytest.mark.parametrize("kind,smoothing,average,nll", LOSSES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}" for c in CASES])
def test_loss_and_gradient(tr, fq, case, dtype, kind, smoothing, average, nll):
    rows, vocab, cu, pad, offset = case
    logits, dev, targets, cu_t, ref_logp = make(rows, vocab, cu, dtype, rows * 7 + vocab, vocab + pad, offset)
    spec = tr.PreferenceLoss(kind, beta=0.3, margin=0.25, label_smoothing=smoothing, average=average, nll_weight=nll)
    out = tr.preference_forward(spec, dev, targets.cuda(), cu_t.cuda(), ref_logp.cuda())
    ref = orc.preference(logits, targets, cu, ref_logp, kind, 0.3, 0.25, smoothing, average, nll)
    row, u, slope, curve = bounds(ref, kind, 0.3, logits, average)
    e = lambda got, want: float((got.cpu().double() - want).abs().max())  # noqa: E731
    n = 1.0 if average else max(1.0, float(ref["counted"].sum()))
    assert e(out.logp, ref["logp"]) <= row
    assert e(out.seq_logp, ref["seq_logp"]) <= row * n + 2.0 ** -24 * float(ref["seq_logp"].abs().max())
    tol = slope * u + (nll * row) + 2.0 ** -22 * float(ref["pair_loss"].abs().max() + 1)
    assert e(out.pair_loss, ref["pair_loss"]) <= tol and e(out.loss, ref["loss"]) <= tol
    # the gradient: coefficient (its own error by the loss's curvature), exp and a quotient; bf16 rounds once more
    amax = torch.zeros(1, device="cuda")
    up = torch.tensor([1.5], device="cuda")
    grad = tr.preference_backward(dev, targets.cuda(), out, dloss=up, amax=amax)
    size = ref["size"] + curve * u * (ref["onehot"] + ref["p"]) * ref["counted"][:, None]
    tol = 1.5 * (orc.type_rounding(dtype) * ref["dlogits"].abs() + 2.0 ** -14 * ref["size"] + 2 * curve * u * (ref["onehot"] + ref["p"])) + 1e-38
    assert ((grad.cpu().double() - 1.5 * ref["dlogits"]).abs() <= tol).all() and size.shape == tol.shape
    assert (grad.cpu()[~ref["counted"]] == 0).all()
    assert amax.item() == grad.float().abs().max().item()
    # the same bits again, into rows of another pitch and offset, and in place
    again = tr.preference_forward(spec, dev, targets.cuda(), cu_t.cuda(), ref_logp.cuda())
    assert torch.equal(again.loss, out.loss) and torch.equal(again.logp, out.logp) and torch.equal(again.dlogp, out.dlogp)
    wide = torch.full((rows, vocab + 5), 7.0, dtype=dtype, device="cuda")
    tr.preference_backward(dev, targets.cuda(), out, dloss=up, dlogits=wide[:, 1:vocab + 1])
    assert torch.equal(wide[:, 1:vocab + 1], grad) and (wide[:, 0] == 7).all() and (wide[:, vocab + 1:] == 7).all()
    alone = tr.preference_forward(spec, dev, targets.cuda(), cu_t.cuda(), ref_logp.cuda(), need_grad=False)
    assert torch.equal(alone.loss, out.loss) and alone.dlogp is None
    seq, logp = tr.sequence_logprob(dev, targets.cuda(), cu_t.cuda(), average=average)
    assert torch.equal(seq, out.seq_logp) and torch.equal(logp, out.logp)
    tr.preference_backward(dev, targets.cuda(), out, dloss=up, dlogits=dev)
    assert torch.equal(dev, grad)
    assert fq.last_device_status() == 0


def test_gradient_against_differences(tr):
    rows, vocab, cu = 12, 40, [0, 3, 7, 9, 12]
    logits, dev, targets, cu_t, ref_logp = make(rows, vocab, cu, torch.float32, 3)
    v = torch.randn((rows, vocab), generator=torch.Generator().manual_seed(5), dtype=torch.float64)
    for kind, smoothing, average, nll in LOSSES:
        spec = tr.PreferenceLoss(kind, 0.3, 0.25, smoothing, average, nll)
        out = tr.preference_forward(spec, dev, targets.cuda(), cu_t.cuda(), ref_logp.cuda())
        grad = orc.d(tr.preference_backward(dev, targets.cuda(), out))
        f = lambda s: float(orc.preference(logits.double() + s * v, targets, cu, ref_logp, kind, 0.3, 0.25, smoothing, average, nll)["loss"])  # noqa: E731
        want = (f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(float((grad * v).sum()) - want) <= 2e-5 * float((grad * v).abs().sum()) + 1e-9


def test_masked_logits(tr):
    """-inf, and the types' lowest value, in the places of tokens that cannot be; a whole row of the lowest value is uniform; NaN and
    infinities in rows that are not counted have no effect; a row that leaves nothing (all -inf) gives a NaN, not a wrong number."""
    for dtype in (torch.bfloat16, torch.float32):
        for vocab in (300, 1029):
            logits, _, targets, cu_t, _ = make(8, vocab, [0, 4, 8], dtype, 9)
            cu = [0, 4, 8]
            targets = torch.randint(0, 10, (8,))
            logits[1, 10:] = float("-inf")
            logits[2, 10:200] = torch.finfo(dtype).min
            logits[3, :] = torch.finfo(dtype).min
            logits[5, :] = torch.finfo(dtype).max
            targets[0] = targets[4] = -1
            logits[0, :] = float("nan")
            logits[4, :7] = float("inf")
            spec = tr.PreferenceLoss(beta=0.1)
            dev = logits.cuda()
            out = tr.preference_forward(spec, dev, targets.cuda(), cu_t.cuda())
            grad = tr.preference_backward(dev, targets.cuda(), out)
            clean = logits.clone()
            clean[0] = clean[4] = 0.0
            ref = orc.preference(clean, targets, cu, None, "sigmoid", 0.1, 0.0, 0.0, False, 0.0)
            assert torch.allclose(out.logp.cpu().double(), ref["logp"], rtol=1e-5, atol=1e-5)
            assert abs(out.loss.item() - float(ref["loss"])) < 1e-5
            assert torch.allclose(grad.cpu().double(), ref["dlogits"], rtol=2 * orc.type_rounding(dtype) + 1e-4, atol=1e-9)
            assert (grad[0] == 0).all() and (grad[4] == 0).all() and (grad[1, 10:] == 0).all()
            logits[6, :] = float("-inf")
            out = tr.preference_forward(spec, logits.cuda(), targets.cuda(), cu_t.cuda())
            assert torch.isnan(out.logp[6]) and torch.isnan(out.loss) and torch.isfinite(out.logp[7])


def test_nothing_counted(tr):
    """Prompts only: log-probabilities and gradients are 0, the loss is that of a margin of 0; with averages, no division by 0."""
    logits, dev, targets, cu_t, _ = make(6, 100, [0, 2, 4, 4, 6], torch.bfloat16, 2)
    targets[:] = -100
    for average in (False, True):
        spec = tr.PreferenceLoss(beta=0.1, average=average, nll_weight=0.5)
        out = tr.preference_forward(spec, dev, targets.cuda(), cu_t.cuda())
        assert (out.seq_logp == 0).all() and (out.logp == 0).all() and abs(out.loss.item() - 0.6931472) < 1e-6
        assert (tr.preference_backward(dev, targets.cuda(), out) == 0).all()


def test_rows_outside_the_sequences_are_not_counted(tr):
    logits, dev, targets, _, _ = make(10, 50, [0, 10], torch.float32, 4)
    targets = torch.randint(0, 50, (10,))
    cu = torch.tensor([2, 4, 7])
    out = tr.preference_forward(tr.PreferenceLoss(), dev, targets.cuda(), cu.cuda())
    grad = tr.preference_backward(dev, targets.cuda(), out)
    assert (out.logp[[0, 1, 7, 8, 9]] == 0).all() and (grad[[0, 1, 7, 8, 9]] == 0).all() and (out.logp[2:7] != 0).all()
    seq, logp = tr.sequence_logprob(dev, targets.cuda(), cu.cuda())
    assert torch.equal(seq, out.seq_logp) and torch.equal(logp, out.logp)


def test_a_target_beyond_the_vocabulary_is_reported(tr, fq):
    logits, dev, targets, cu_t, _ = make(6, 100, [0, 3, 6], torch.float32, 6)
    targets[5] = 100
    assert fq.last_device_status() == 0
    out = tr.preference_forward(tr.PreferenceLoss(), dev, targets.cuda(), cu_t.cuda())
    grad = tr.preference_backward(dev, targets.cuda(), out)
    assert fq.last_device_status() == fq.ERR_INVALID_ARG and fq.last_device_status() == 0
    assert out.logp[5] == 0 and (grad[5] == 0).all() and torch.isfinite(out.loss)


def test_extreme_margins(tr):
    """Differences far beyond the range of exp give the limits, not NaN."""
    logits, dev, targets, cu_t, _ = make(4, 64, [0, 2, 4], torch.float32, 8)
    for ref in ([1e6, -1e6], [-1e6, 1e6]):
        for kind in ("sigmoid", "hinge"):
            out = tr.preference_forward(tr.PreferenceLoss(kind, beta=10.0), dev, targets.cuda(), cu_t.cuda(), torch.tensor(ref).cuda())
            grad = tr.preference_backward(dev, targets.cuda(), out)
            assert torch.isfinite(out.loss) and torch.isfinite(grad).all()
            assert (out.loss.item() > 1e6) == (ref[0] > 0)
            assert (grad.abs().max().item() > 0) == (ref[0] > 0)


def test_many_pairs(tr):
    """More pairs than threads of the block that takes the mean."""
    pairs = 700
    rows = 2 * pairs
    logits, dev, targets, cu_t, ref_logp = make(rows, 33, list(range(rows + 1)), torch.float32, 12)
    out = tr.preference_forward(tr.PreferenceLoss(), dev, targets.cuda(), cu_t.cuda(), ref_logp.cuda())
    ref = orc.preference(logits, targets, list(range(rows + 1)), ref_logp, "sigmoid", 0.1, 0.0, 0.0, False, 0.0)
    assert abs(out.loss.item() - float(ref["loss"])) < 1e-6
    assert float((out.pair_loss.cpu().double() - ref["pair_loss"]).abs().max()) < 1e-5


def test_another_stream_and_a_captured_graph(tr):
    logits, dev, targets, cu_t, ref_logp = make(64, 5000, [0, 10, 30, 50, 64], torch.bfloat16, 10)
    args = (targets.cuda(), cu_t.cuda(), ref_logp.cuda())
    spec = tr.PreferenceLoss(beta=0.2)
    out = tr.preference_forward(spec, dev, *args)
    want = tr.preference_backward(dev, args[0], out)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o = tr.preference_forward(spec, dev, *args)
        g = tr.preference_backward(dev, args[0], o)
    side.synchronize()
    assert torch.equal(o.loss, out.loss) and torch.equal(g, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = tr.preference_forward(spec, dev, *args)
        g = tr.preference_backward(dev, args[0], o)
    for _ in range(3):
        g.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o.loss, out.loss) and torch.equal(g, want)


def test_offsets_beyond_32_bits(tr):
    """More than 2^31 logits: the last rows lie where a 32-bit offset would wrap."""
    rows, vocab = 16400, 131072                       # 2.15e9 values
    dev = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
    dev[-1, 5] = 8.0
    targets = torch.full((rows,), -100, dtype=torch.int64, device="cuda")
    targets[-1], targets[0] = 5, 7
    cu = torch.tensor([0, 8000, rows], device="cuda")
    out = tr.preference_forward(tr.PreferenceLoss(beta=1.0), dev, targets, cu)
    import math
    assert abs(out.logp[-1].item() - (8.0 - math.log(math.exp(8.0) + vocab - 1))) < 1e-4
    assert abs(out.logp[0].item() + math.log(vocab)) < 1e-4
    tr.preference_backward(dev, targets, out, dlogits=dev)
    c = out.dlogp[-1].item()
    p = math.exp(out.logp[-1].item())
    assert abs(dev[-1, 5].item() - c * (1 - p)) < 2 ** -8 * abs(c) and dev[1:-1].abs().max().item() == 0
