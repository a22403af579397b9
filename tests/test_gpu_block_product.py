"""The products of a layer held in 8 bits by blocks, against the codes' values multiplied in 64 bits.

Tolerance.  The codes' values are exact, products of two codes too.  An instruction adds 32 products to an fp32 accumulator, each
addition off by at most 2^-22 of the sum of sizes so far (two units in the last place, for an alignment that cuts off instead of
rounding), so K / 32 of them are off by at most (K / 32 + 1) * 2^-22 * sum |a| |b|; then the result's rounding, half a step."""
import pytest
import torch

from tests import dense_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def data(rows, cols, seed, loud=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, device="cuda")
    if loud:       # scales that differ from block to block, in both directions
        x *= torch.exp2(torch.randint(-8, 8, (-(-rows // 32), -(-cols // 64)), generator=g, device="cuda").float()).repeat_interleave(32, 0)[:rows].repeat_interleave(64, 1)[:, :cols]
    return x


def close(got, a, b):
    """got against a @ b, both in 64 bits."""
    want, size = a @ b, a.abs() @ b.abs()
    k = a.shape[1]
    bound = (k / 32 + 1) * 2.0 ** -22 * size + torch.finfo(got.dtype).eps / 2 * want.abs() * (1 + 2.0 ** -10)
    over = (got.double() - want).abs() > bound
    assert not over.any(), (int(over.sum()), over.nonzero()[:4].tolist(), float(((got.double() - want).abs() / bound.clamp(min=1e-300)).max()))


SIZES = [(1, 16, 16), (1, 128, 128), (7, 144, 272), (128, 128, 256), (200, 1040, 528), (256, 512, 256), (300, 2064, 1040), (513, 640, 4112),
         (64, 4096, 1024), (1000, 528, 2000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,n,m", SIZES)
def test_forward(dense, T, n, m, dtype):
    x, w = dense.block_quantize(data(T, n, 1), "row"), dense.block_quantize(data(m, n, 2), "tile")
    close(dense.block_forward(x, w, dtype), orc.value(x), orc.value(w).T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,n,m", SIZES)
def test_input_grad(dense, T, n, m, dtype):
    dy, w = dense.block_quantize(data(T, m, 3), "row", "e5m2"), dense.block_quantize(data(m, n, 4), "tile")
    close(dense.block_input_grad(dy, w, dtype), orc.value(dy), orc.value(w))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,n,m", SIZES)
def test_weight_grad(dense, T, n, m, dtype):
    dy, x = dense.block_quantize(data(T, m, 5), "col", "e5m2"), dense.block_quantize(data(T, n, 6), "col")
    close(dense.block_weight_grad(dy, x, dtype), orc.value(dy).T, orc.value(x))


@pytest.mark.parametrize("way,T,n,m", [("dw", 16500, 2064, 2000), ("dw", 8193, 2064, 2000), ("fwd", 2100, 8320, 2064), ("dx", 2100, 2064, 16400)])
def test_long_contraction_in_fp32(dense, way, T, n, m):
    """Parts of 8192 terms, each off as above by at most 257 * 2^-22 of its own sum of sizes, and ordinary additions of up to three of them,
    each off by at most half a step of what is then there: 3 * 2^-24 of the whole sum of sizes, with a tenth to spare."""
    if way == "dw":
        dy, x = dense.block_quantize(data(T, m, 41), "col", "e5m2"), dense.block_quantize(data(T, n, 42), "col")
        got, a, b = dense.block_weight_grad(dy, x, torch.float32), orc.value(dy).T, orc.value(x)
    elif way == "fwd":
        x, w = dense.block_quantize(data(T, n, 43), "row"), dense.block_quantize(data(m, n, 44), "tile")
        got, a, b = dense.block_forward(x, w, torch.float32), orc.value(x), orc.value(w).T
    else:
        dy, w = dense.block_quantize(data(T, m, 45), "row", "e5m2"), dense.block_quantize(data(m, n, 46), "tile")
        got, a, b = dense.block_input_grad(dy, w, torch.float32), orc.value(dy), orc.value(w)
    off, size = (got.double() - a @ b).abs(), a.abs() @ b.abs()
    bound = (257 * 2.0 ** -22 + 3 * 2.0 ** -24 * 1.1) * size
    assert not (off > bound).any(), (int((off > bound).sum()), float((off / bound.clamp(min=1e-300)).max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("x_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,n,m", SIZES + [(2, 4096, 4096), (5, 11008, 512), (16, 2064, 1040), (19, 2064, 1040), (33, 512, 512)])
def test_linear(dense, T, n, m, x_dtype, dtype):
    x, w = data(T, n, 7).to(x_dtype), dense.block_quantize(data(m, n, 8), "tile")
    v, e = orc.quantize(x, "row", "e4m3")
    a = v * torch.exp2(orc.spread(e, "row", T, n).double() - 127.0)
    close(dense.block_forward(x, w, dtype), a, orc.value(w).T)


@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
def test_formats(dense, formats):
    fa, fb = formats
    T, n, m = 260, 400, 528
    x, w, dy = dense.block_quantize(data(T, n, 1), "row", fa), dense.block_quantize(data(m, n, 2), "tile", fb), dense.block_quantize(data(T, m, 3), "row", fa)
    close(dense.block_forward(x, w, torch.float32), orc.value(x), orc.value(w).T)
    close(dense.block_input_grad(dy, w, torch.float32), orc.value(dy), orc.value(w))
    a, b = dense.block_quantize(data(T, m, 3), "col", fa), dense.block_quantize(data(T, n, 1), "col", fb)
    close(dense.block_weight_grad(a, b, torch.float32), orc.value(a).T, orc.value(b))


@pytest.mark.parametrize("T", [3, 300])
def test_nan_blocks(dense, T):
    """A NaN block makes NaN of the rows (columns) it takes part in, and of nothing else."""
    n, m = 528, 400
    x, w = data(T, n, 1), data(m, n, 2)
    x[2, 300], w[130, 5] = float("nan"), float("inf")
    for y in (dense.block_forward(dense.block_quantize(x), dense.block_quantize(w, "tile"), torch.float32),
              dense.block_forward(x, dense.block_quantize(w, "tile"), torch.float32)):
        bad = torch.zeros((T, m), dtype=torch.bool, device="cuda")
        bad[2] = True
        bad[:, 128:256] = True
        assert torch.equal(torch.isnan(y), bad)


def test_extreme_scales(dense):
    """Scales at both ends of their range, whose product is a normal number."""
    T, n, m = 40, 256, 64
    x, w = torch.full((T, n), 2.0 ** 120, device="cuda"), torch.full((m, n), 2.0 ** -125, device="cuda")
    for y in (dense.block_forward(dense.block_quantize(x), dense.block_quantize(w, "tile"), torch.float32), dense.block_forward(x[:2], dense.block_quantize(w, "tile"), torch.float32)):
        assert (y == 2.0 ** -5 * n).all()
    z = dense.block_forward(torch.zeros((T, n), device="cuda"), dense.block_quantize(w, "tile"), torch.float32)
    assert (z == 0).all()
