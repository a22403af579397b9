"""8-bit codes by blocks of 128: codes and scale bytes against the definition in 64 bits, bit for bit."""
import pytest
import torch

from tests import dense_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def tensor(rows, cols, dtype, seed=0):
    """Values whose size changes over the tensor, with zeros, a zero block and values at the border of a scale."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g, device="cuda").float())
    x[torch.rand((rows, cols), generator=g, device="cuda") < 0.05] = 0.0
    x[: rows // 3, : min(cols, 130)] = 0.0
    x[-1, -1] = 448.0
    if rows > 1:
        x[-2, 0] = 449.0
    return x.to(dtype)


def check(q, x, along, fmt):
    v, e = orc.quantize(x, along, fmt)
    assert q.codes.dtype == orc.TYPES[fmt] and q.along == along
    assert torch.equal(q.scales, e)
    got = q.codes.double()
    assert torch.equal(torch.isnan(got), torch.isnan(v)) and torch.equal(got.nan_to_num(0.0), v.nan_to_num(0.0))


SIZES = [(1, 1), (1, 16), (1, 4096), (2, 127), (3, 128), (128, 128), (129, 136), (127, 129), (300, 1000), (257, 1011), (16, 5), (1000, 8), (130, 2064)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_codes_and_scales(dense, rows, cols, dtype, fmt):
    x = tensor(rows, cols, dtype)
    for along in ("row", "col", "tile"):
        check(dense.block_quantize(x, along, fmt), x, along, fmt)
    row, col = dense.block_quantize_both(x, fmt)
    check(row, x, "row", fmt)
    check(col, x, "col", fmt)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("along", ["row", "col", "tile"])
def test_infinities_nan_and_extremes(dense, along, dtype):
    x = tensor(300, 400, dtype, 3)
    x[5, 7], x[5, 200], x[200, 300] = float("inf"), float("nan"), float("-inf")
    x[140:270, 130:260] = torch.finfo(dtype).max
    x[270:300, 0:128] = torch.finfo(dtype).tiny
    x[271, 3] = torch.finfo(dtype).smallest_normal / 8 if dtype == torch.float32 else 0.0
    for fmt in ("e4m3", "e5m2"):
        check(dense.block_quantize(x, along, fmt), x, along, fmt)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,pitch", [(0, 512), (1, 512), (8, 520), (0, 391), (3, 1001)])
def test_row_pitch_and_alignment(dense, dtype, offset, pitch):
    big = tensor(200, 1 + pitch, dtype, 5).flatten()
    x = torch.as_strided(big, (150, 384), (pitch, 1), offset)
    for along in ("row", "col", "tile"):
        check(dense.block_quantize(x, along), x, along, "e4m3")


@pytest.mark.parametrize("along", ["row", "col", "tile"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (130, 300), (257, 1011), (5, 4096)])
def test_dequantize(dense, rows, cols, fmt, along):
    x = tensor(rows, cols, torch.float32, 7)
    if rows > 3:
        x[2, 1] = float("nan")
    q = dense.block_quantize(x, along, fmt)
    want = orc.value(q)
    for dtype in (torch.float32, torch.bfloat16):
        got = dense.block_dequantize(q, dtype)
        assert torch.equal(got.nan_to_num(7.0), want.to(dtype).nan_to_num(7.0))


def test_out_and_refusals(dense):
    x = torch.randn((64, 256), device="cuda")
    q = dense.block_quantize(x)
    again = dense.block_quantize(2 * x, out=q)
    assert again.codes.data_ptr() == q.codes.data_ptr() and int((again.scales.int() - dense.block_quantize(x).scales.int()).unique()) == 1
    for bad in (dict(along="diagonal"), dict(fmt="e3m4"), dict(out=dense.block_quantize(x, "col")), dict(out=dense.block_quantize(x, fmt="e5m2"))):
        with pytest.raises(ValueError):
            dense.block_quantize(x, **bad)
    with pytest.raises(ValueError):
        dense.block_quantize(x.T)
    with pytest.raises(ValueError):
        dense.block_quantize(x[:0])
    with pytest.raises(TypeError):
        dense.block_quantize(x.half())
    with pytest.raises(ValueError):
        dense.block_dequantize(q._replace(scales=q.scales[:-1]))
