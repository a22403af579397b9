"""fp32 results of long contractions: the tensor core's additions cut off, so what is summed in tensor memory is no longer than 2048 terms,
however a tile's contraction is shared.

Tolerances.  Element by element, signs random: parts of 2048 terms, each off by at most 65 * 2^-22 of its own sum of sizes (the products' tests
derive it), and an ordinary addition for each part, off by at most half a step of what is then there.
Of the norm, all values positive, so that nothing that is cut off makes up for anything: an instruction adds 32 products to a sum and cuts off
less than a step, 2^-23 of it.  Of equally many terms each, the sums before the end of a part are on average half of it, so 64 instructions lose at
most 32.5 * 2^-23 = 3.9e-6 of a part and of the whole, and n ordinary additions of equal parts at most n / 2 * 2^-24.
Of the norm, signs random, scales that differ from block to block: the sums before the end of a part are in size two thirds of it (the square root's
average), a step is on average 0.72 * 2^-23 of a sum, and half a step is cut off on average, always towards zero: 64 * 2/3 * 0.72 / 2 * 2^-23 =
1.8e-6 of a part, and no more of the whole.  (Parts of 8192 terms would leave four times as much.)"""
import pytest
import torch

from tests import dense_oracle as orc
from tests.test_gpu_block_product import data

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


SIZES = [("dw", 65536, 1024, 256), ("dw", 131072, 1024, 256), ("dw", 131072 - 500, 1040, 272), ("dw", 65536, 1024, 2048), ("dw", 98304, 528, 16),
         ("dw", 100000, 2064, 400), ("fwd", 64, 131072, 1024), ("fwd", 300, 100000, 528), ("dx", 64, 1024, 131072), ("dx", 5, 2064, 65552)]


def product(dense, way, T, n, m, positive):
    """(result, its operands in 64 bits)"""
    make = lambda rows, cols, seed: data(rows, cols, seed, False).abs() if positive else data(rows, cols, seed, False)  # noqa: E731
    if way == "dw":
        dy, x = dense.block_quantize(make(T, m, 51), "col"), dense.block_quantize(make(T, n, 52), "col")
        return dense.block_weight_grad(dy, x, torch.float32), orc.value(dy).T, orc.value(x)
    if way == "fwd":
        x, w = dense.block_quantize(make(T, n, 53), "row"), dense.block_quantize(make(m, n, 54), "tile")
        return dense.block_forward(x, w, torch.float32), orc.value(x), orc.value(w).T
    dy, w = dense.block_quantize(make(T, m, 55), "row"), dense.block_quantize(make(m, n, 56), "tile")
    return dense.block_input_grad(dy, w, torch.float32), orc.value(dy), orc.value(w)


@pytest.mark.parametrize("way,T,n,m", SIZES)
def test_shared_contraction_in_parts(dense, way, T, n, m):
    got, a, b = product(dense, way, T, n, m, True)
    want = a @ b
    parts = -(-a.shape[1] // 2048) + 4        # (a pair's last part may be short)
    off = float((got.double() - want).norm() / want.norm())
    assert off <= 3.9e-6 + parts / 2 * 2.0 ** -24, off
    got, a, b = product(dense, way, T, n, m, False)
    size = a.abs() @ b.abs()
    assert not ((got.double() - a @ b).abs() > (65 * 2.0 ** -22 + parts * 2.0 ** -24 * 1.1) * size).any()


@pytest.mark.parametrize("way,T,n,m", [("dw", 8192, 1040, 2064), ("dw", 16384, 2048, 4096), ("fwd", 1000, 11008, 2064), ("fwd", 8, 11008, 4096), ("fwd", 300, 8192, 528),
                                       ("dx", 1000, 2064, 11008), ("dx", 777, 5120, 13824), ("dw", 65536, 1024, 256)])
def test_scales_that_differ(dense, way, T, n, m):
    if way == "dw":
        dy, x = dense.block_quantize(data(T, m, 57), "col"), dense.block_quantize(data(T, n, 58), "col")
        got, a, b = dense.block_weight_grad(dy, x, torch.float32), orc.value(dy).T, orc.value(x)
    elif way == "fwd":
        x, w = dense.block_quantize(data(T, n, 57), "row"), dense.block_quantize(data(m, n, 58), "tile")
        got, a, b = dense.block_forward(x, w, torch.float32), orc.value(x), orc.value(w).T
    else:
        dy, w = dense.block_quantize(data(T, m, 57), "row"), dense.block_quantize(data(m, n, 58), "tile")
        got, a, b = dense.block_input_grad(dy, w, torch.float32), orc.value(dy), orc.value(w)
    want = a @ b
    assert float((got.double() - want).norm() / want.norm()) <= 1.8e-6, float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("T,n,m", [(40000, 1040, 272), (70001, 528, 16), (50000, 1040, 656)])
def test_passes_by_themselves_and_together(dense, T, n, m):
    """The kernel of several passes between margins, the same bits twice, captured and replayed over new inputs, on two streams at once."""
    from tests.test_gpu_train_guard_bands import fence, finish
    make = lambda seed: (dense.block_quantize(data(T, m, seed, False), "col"), dense.block_quantize(data(T, n, seed + 1, False), "col"))  # noqa: E731
    a, b = make(61), make(63)
    p = lambda q: (q.codes.data_ptr(), q.scales.data_ptr(), 0)  # noqa: E731
    out = fence(o=((m, n), torch.float32))
    finish(dense.lib.falqon_block_weight_grad(*p(a[0]), *p(a[1]), T, n, m, out["o"].p, 1, None), out, T=T, n=n, m=m)
    want = [dense.block_weight_grad(*a), dense.block_weight_grad(*b)]
    assert torch.equal(out["o"].t, want[0]) and torch.equal(dense.block_weight_grad(*a), want[0])
    held = [dense.Blocks(q.codes.clone(), q.scales.clone(), q.along) for q in a]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = dense.block_weight_grad(*held)
    for source, w in ((a, want[0]), (b, want[1])):
        for h, q in zip(held, source):
            h.codes.copy_(q.codes)
            h.scales.copy_(q.scales)
        graph.replay()
        assert torch.equal(got, w)
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(4):
        for s, mine, q in zip(streams, results, (a, b)):
            with torch.cuda.stream(s):
                mine.append(dense.block_weight_grad(*q))
    torch.cuda.synchronize()
    assert all(torch.equal(r, w) for mine, w in zip(results, want) for r in mine)


def test_a_nan_block_in_a_later_pass(dense):
    T, n, m = 60000, 528, 144
    x, dy = data(T, n, 71, False), data(T, m, 72, False)
    x[T - 5, 300], dy[T // 2, 17] = float("nan"), float("inf")
    got = dense.block_weight_grad(dense.block_quantize(dy, "col"), dense.block_quantize(x, "col"))
    bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    bad[17], bad[:, 300] = True, True
    assert torch.equal(torch.isnan(got), bad)
