"""The calls of dense.py as a program makes them: one after the other in a training step, captured and replayed, on two streams at once, the
same bits twice, beyond 32-bit offsets; and which kernels their rules choose."""
import ctypes as C

import pytest
import torch

from tests import dense_oracle as orc
from tests.launches import launched

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def whole(shape, most, seed):
    """Whole numbers: exact in 8 bits (up to 16) under any scale of a block that holds `most`, so that every product and sum is exact."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").float()


@pytest.mark.parametrize("T,n,m", [(3, 144, 272), (200, 272, 400), (700, 528, 1040)])
def test_gradients_are_differences(dense, T, n, m):
    """The layer is linear in x and in w, so its gradients are its differences, exactly where the numbers are whole ones: with
    L = sum(r * (x w^T)), L(x + d) - L(x) = sum(dx * d) and L(w + e) - L(w) = sum(dw * e)."""
    x, d, w, e, r = (whole(s, 3, i) for i, s in enumerate(((T, n), (T, n), (m, n), (m, n), (T, m))))
    loss = lambda a, b: (r.double() * dense.block_forward(dense.block_quantize(a), dense.block_quantize(b, "tile"), torch.float32).double()).sum()  # noqa: E731
    (rr, rc), xc, wt = dense.block_quantize_both(r), dense.block_quantize(x, "col"), dense.block_quantize(w, "tile")
    dx, dw = dense.block_input_grad(rr, wt, torch.float32), dense.block_weight_grad(rc, xc)
    assert torch.equal(dx, r @ w) and torch.equal(dw, r.T @ x)
    assert loss(x + d, w) - loss(x, w) == (dx.double() * d.double()).sum()
    assert loss(x, w + e) - loss(x, w) == (dw.double() * e.double()).sum()


def step(dense, x, dy, w, momentum, lr=0.02):
    """A step of one layer trained in 8 bits by blocks: forward, both gradients, momentum, orthogonalised update, weights quantized again."""
    wt = dense.block_quantize(w, "tile")
    xr, xc = dense.block_quantize_both(x)
    y = dense.block_forward(xr, wt)
    gr, gc = dense.block_quantize_both(dy)
    dx, dw = dense.block_input_grad(gr, wt), dense.block_weight_grad(gc, xc)
    momentum = momentum * 0.95 + dw
    o = dense.orthogonalize(momentum, scale=0.2 * max(w.shape) ** 0.5)
    w = w - lr * o
    return y, dx, dw, momentum, o, w, dense.block_quantize(w, "tile")


@pytest.mark.parametrize("T,n,m", [(70, 272, 144), (513, 400, 656), (300, 1040, 64)])
def test_a_training_step(dense, T, n, m):
    """Each result against 64 bits from the codes that the step itself made; the products' bound as in their own test, the update's too."""
    g = torch.Generator(device="cuda").manual_seed(T)
    x, dy = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((T, n), (T, m)))
    w, momentum = torch.randn((m, n), generator=g, device="cuda") * 0.02, torch.randn((m, n), generator=g, device="cuda") * 0.1
    y, dx, dw, mom, o, w2, wq = step(dense, x, dy, w, momentum)

    def q(t, along):
        v, e = orc.quantize(t, along, "e4m3")
        return v * torch.exp2(orc.spread(e, along, *t.shape).double() - 127.0)

    for got, a, b in ((y, q(x, "row"), q(w, "tile").T), (dx, q(dy, "row"), q(w, "tile")), (dw, q(dy, "col").T, q(x, "col"))):
        bound = (a.shape[1] / 32 + 1) * 2.0 ** -22 * (a.abs() @ b.abs()) + torch.finfo(got.dtype).eps / 2 * (a @ b).abs() * (1 + 2.0 ** -10)
        assert ((got.double() - a @ b).abs() <= bound).all()
    want = orc.orthogonalize(mom, [orc.QUINTIC] * 5, 1e-7, 0.2 * max(m, n) ** 0.5)
    assert float((o.double() - want).norm() / want.norm()) <= 1e-5
    v, e = orc.quantize(w2, "tile", "e4m3")
    assert torch.equal(wq.scales, e) and torch.equal(wq.codes.double(), v)


def test_same_bits_twice(dense):
    g = torch.Generator(device="cuda").manual_seed(0)
    x, dy, w, mom = (torch.randn(s, generator=g, device="cuda") for s in ((300, 1040), (300, 656), (656, 1040), (656, 1040)))
    first = step(dense, x, dy, w, mom)
    for _ in range(3):
        for a, b in zip(first[:-1], step(dense, x, dy, w, mom)):
            assert torch.equal(a, b)
    for shape in ((7, 700, 64), (2, 100, 3000), (1, 130, 900)):
        u = torch.randn(shape, generator=g, device="cuda")
        for dtype in (torch.bfloat16, torch.float32):
            a = dense.orthogonalize(u, dtype=dtype)
            assert all(torch.equal(a, dense.orthogonalize(u, dtype=dtype)) for _ in range(3))


def test_captured_steps(dense):
    """Two steps captured from one pool, replayed in turn and over new inputs: what eager calls give."""
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda: [torch.randn(s, generator=g, device="cuda") for s in ((257, 528), (257, 400), (400, 528), (400, 528))]  # noqa: E731
    held = [new(), new()]
    one = torch.randn((1, 528), generator=g, device="cuda").bfloat16()
    for h in held:
        step(dense, *h)
    torch.cuda.synchronize()
    graphs, outs, pool = [], [], torch.cuda.graph_pool_handle()
    for h in held:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            r = step(dense, *h)
            outs.append((r, dense.block_forward(one, r[-1])))
        graphs.append(graph)
    for _ in range(3):
        for h in held:
            for t, v in zip(h, new()):
                t.copy_(v)
        for k in (0, 1):
            graphs[k].replay()
            got = [t.clone() for t in outs[k][0][:-1]] + [outs[k][1].clone()]
            want = step(dense, *held[k])
            for a, b in zip(got, [*want[:-1], dense.block_forward(one, want[-1])]):
                assert torch.equal(a, b)


def test_two_streams_at_once(dense):
    """The same weights on two streams, calls of both in flight together."""
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.randn((1040, 2064), generator=g, device="cuda") * 0.02
    xs = [torch.randn((T, 2064), generator=g, device="cuda").bfloat16() for T in (1, 300)]
    ups = [torch.randn(s, generator=g, device="cuda") for s in ((4, 64, 3000), (300, 700))]
    wt = dense.block_quantize(w, "tile")
    want = [[dense.block_forward(x, wt) for x in xs] + [dense.orthogonalize(u) for u in ups] for _ in range(2)][0]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(5):
        for s, mine in zip(streams, got):
            with torch.cuda.stream(s):
                mine.append([dense.block_forward(x, wt) for x in xs] + [dense.orthogonalize(u) for u in ups])
    torch.cuda.synchronize()
    for mine in got:
        for r in mine:
            assert all(torch.equal(a, b) for a, b in zip(r, want))
    from paper_2510_24061_b200 import binding as fq
    assert fq.last_device_status() == 0


def test_beyond_32_bit_offsets(dense):
    """More than 2^32 values: the last rows and columns come out as they do by themselves."""
    rows, cols = 131200, 32768 + 16
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((256, cols), device="cuda").bfloat16()
    x[-256:] = tail              # 131200 is a multiple of 128: the tail's blocks are the tensor's
    for along in ("row", "col", "tile"):
        q, t = dense.block_quantize(x, along), dense.block_quantize(tail, along)
        assert torch.equal(q.codes[-256:].view(torch.uint8), t.codes.view(torch.uint8))
        assert torch.equal(q.scales[-t.scales.shape[0]:], t.scales)
        assert torch.equal(dense.block_dequantize(q)[-256:], dense.block_dequantize(t))
        del q
    for T in (2, 40):            # as weights: both kernels of the forward, and the input gradient, whose contraction passes 2^32
        wt = dense.block_quantize(x, "tile")
        part = orc.value(dense.block_quantize(tail, "tile"))
        a = dense.block_quantize(torch.randn((T, cols), device="cuda"))
        y = dense.block_forward(a, wt)
        within(y[:, -256:], orc.value(a), part.T)
        assert not y[:, :-256].any()
        dy = torch.zeros((T, rows), device="cuda")
        dy[:, -256:] = torch.randn((T, 256), device="cuda")
        within(dense.block_input_grad(dense.block_quantize(dy), wt), orc.value(dense.block_quantize(dy[:, -256:].contiguous())), part)
        del wt


def within(got, a, b):
    """got against a @ b, by the bound that the products' tests derive.  (The same numbers in a tensor of another shape may be added up in
    another order: a short contraction's tile may be one CTA pair's, or shared by four.)"""
    want, size = a @ b, a.abs() @ b.abs()
    bound = (a.shape[1] / 32 + 1) * 2.0 ** -22 * size + torch.finfo(got.dtype).eps / 2 * want.abs() * (1 + 2.0 ** -10)
    assert ((got.double() - want).abs() <= bound).all()


def test_beyond_32_bit_offsets_of_a_batch(dense):
    batch, rows, cols = 260, 4096, 4096 + 8
    g = torch.zeros((batch, rows, cols), dtype=torch.bfloat16, device="cuda")
    g[-1] = torch.randn((rows, cols), device="cuda")
    out = dense.orthogonalize(g)
    assert torch.equal(out[-1], dense.orthogonalize(g[-1])) and not out[:-1].any()


def names(call):
    return [n for n, *_ in launched(call)]


def test_which_kernels_run(dense):
    """Both sides of each rule's border, read from captured graphs."""
    w = dense.block_quantize(torch.randn((512, 1024), device="cuda"), "tile")
    x = torch.randn((64, 1024), device="cuda").bfloat16()
    few = names(lambda: dense.block_forward(x[:4], w))
    assert len(few) == 1 and "block_linear" in few[0]
    more = names(lambda: dense.block_forward(x[:5], w))
    assert len(more) == 2 and "block_quant_kernel" in more[0] and "block_product" in more[1]
    large = dense.block_quantize(torch.zeros((32768 + 16, 1024), device="cuda"), "tile")          # just over 2^25 weights
    assert len(names(lambda: dense.block_forward(x[:2], large))) == 1 and len(names(lambda: dense.block_forward(x[:3], large))) == 2
    q = dense.block_quantize(x[:4].contiguous())
    assert "block_linear" in names(lambda: dense.block_forward(q, w))[0]
    assert "block_product" in names(lambda: dense.block_forward(dense.block_quantize(x[:5].contiguous()), w))[-1]
    assert "block_quant_kernel" in names(lambda: dense.block_quantize(x))[0]
    assert "ragged" in names(lambda: dense.block_quantize(x[:, 1:]))[0] and "ragged" in names(lambda: dense.block_quantize(x[:, :1023]))[0]
    for shape, dtype, thin in (((64, 900), torch.bfloat16, True), ((65, 900), torch.bfloat16, False), ((900, 128), torch.float32, True), ((900, 129), torch.float32, False)):
        ran = names(lambda: dense.orthogonalize(torch.ones(shape, device="cuda", dtype=dtype)))
        assert ("thin_gram" in ran[-3]) == thin, ran
    # more steps than fp64 digits allow from the Gram matrix
    assert "thin" not in names(lambda: dense.orthogonalize(torch.ones((64, 900), device="cuda"), steps=9))[-1]
    assert "thin" in names(lambda: dense.orthogonalize(torch.ones((64, 900), device="cuda"), steps=8))[-1]


def test_rows_that_do_not_fill_a_tile_go_their_own_way(dense):
    """777 rows over a long contraction: three tiles of 256, and a launch for the nine rows behind them; each within the products' bound."""
    T, n, m = 777, 5120, 13824
    g = torch.Generator(device="cuda").manual_seed(4)
    w = dense.block_quantize(torch.randn((m, n), generator=g, device="cuda"), "tile")
    dy = dense.block_quantize(torch.randn((T, m), generator=g, device="cuda") * torch.exp2(torch.arange(T, device="cuda") % 9 - 4.0)[:, None])
    ran = names(lambda: dense.block_input_grad(dy, w))
    assert len(ran) == 2 and all("block_product" in k for k in ran), ran
    for dtype in (torch.bfloat16, torch.float32):
        within(dense.block_input_grad(dy, w, dtype), orc.value(dy), orc.value(w))
