"""Every buffer that a call of include/falqon_dense.h may write lies between margins of a pattern: none is touched, at sizes whose last
vectors, blocks, tiles and pieces are partial; and what a call does not own is not written."""
import ctypes as C

import pytest
import torch

from tests.test_gpu_train_guard_bands import Fenced, fence, finish

pytestmark = pytest.mark.gpu
u8, f32 = torch.uint8, torch.float32


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 127), (127, 129), (128, 128), (130, 264), (257, 1011), (5, 4096), (300, 2064)])
def test_quantizer(dense, rows, cols, dtype):
    code, nr, nc = (0 if dtype == torch.bfloat16 else 1), -(-rows // 128), -(-cols // 128)
    x = torch.randn((rows, cols), device="cuda").to(dtype)
    for along, shape in ((0, (rows, nc)), (1, (nr, cols)), (2, (nr, nc))):
        out = fence(c=((rows, cols), u8), s=(shape, u8))
        finish(dense.lib.falqon_block_quantize(x.data_ptr(), code, rows, cols, cols, 0, along, out["c"].p, out["s"].p, None), out, rows=rows, cols=cols, along=along)
        back = fence(y=((rows, cols), dtype))
        finish(dense.lib.falqon_block_dequantize(out["c"].p, out["s"].p, 0, along, rows, cols, back["y"].p, code, None), back, rows=rows, cols=cols, along=along)
    both = fence(rc=((rows, cols), u8), rs=((rows, nc), u8), cc=((rows, cols), u8), cs=((nr, cols), u8))
    finish(dense.lib.falqon_block_quantize_both(x.data_ptr(), code, rows, cols, cols, 0, both["rc"].p, both["rs"].p, both["cc"].p, both["cs"].p, None), both,
           rows=rows, cols=cols)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,n,m", [(1, 16, 16), (3, 144, 272), (4, 2064, 1040), (7, 528, 400), (130, 272, 144), (257, 656, 1296), (513, 128, 2064)])
def test_products(dense, T, n, m, dtype):
    code = 0 if dtype == torch.bfloat16 else 1
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w, dy = (torch.randn(s, generator=g, device="cuda") for s in ((T, n), (m, n), (T, m)))
    (xr, xc), (gr, gc), wt = dense.block_quantize_both(x), dense.block_quantize_both(dy), dense.block_quantize(w, "tile")
    p = lambda q: (q.codes.data_ptr(), q.scales.data_ptr(), 0)  # noqa: E731
    for name, a, b, shape in (("forward", xr, wt, (T, m)), ("input_grad", gr, wt, (T, n)), ("weight_grad", gc, xc, (m, n))):
        out = fence(o=(shape, dtype))
        finish(getattr(dense.lib, f"falqon_block_{name}")(*p(a), *p(b), T, n, m, out["o"].p, code, None), out, what=name, T=T, n=n, m=m)
    xd = x.to(dtype)
    size = dense.lib.falqon_block_linear_scratch_bytes(T, n, m)
    out = fence(y=((T, m), dtype), ws=((max(size, 1),), u8))
    finish(dense.lib.falqon_block_linear(xd.data_ptr(), code, *p(wt), T, n, m, out["y"].p, code, out["ws"].p, size, None), out, what="linear", T=T, n=n, m=m)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (1, 7, 3), (2, 33, 70), (3, 500, 17), (2, 129, 130), (1, 257, 1000), (1, 1000, 300), (5, 64, 512), (1, 128, 4096),
                                             (1, 4100, 130)])
def test_orthogonalize(dense, batch, rows, cols, dtype):
    code = 0 if dtype == torch.bfloat16 else 1
    g = torch.randn((batch, rows, cols), device="cuda").to(dtype)
    for out_dtype in (torch.bfloat16, torch.float32):
        plan = dense.falqon_ortho(batch, rows, cols, code, 0 if out_dtype == torch.bfloat16 else 1, 5, 1e-7, 1.0, None)
        size = dense.lib.falqon_orthogonalize_scratch_bytes(C.byref(plan))
        out = fence(o=((batch, rows, cols), out_dtype), ws=((size,), u8))
        before = g.clone()
        finish(dense.lib.falqon_orthogonalize(C.byref(plan), g.data_ptr(), out["o"].p, out["ws"].p, size, None), out, batch=batch, rows=rows, cols=cols)
        assert torch.equal(g, before) and torch.isfinite(out["o"].t).all()
