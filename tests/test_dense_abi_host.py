"""Host-side checks of include/falqon_dense.h that need no GPU: exported symbols, plain C, sizes, refusals before any launch."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000      # an aligned non-null address that is never dereferenced on these paths


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import build
    build.build()
    from paper_2510_24061_b200 import dense
    return dense


@pytest.fixture(scope="module")
def fq(dense):
    from paper_2510_24061_b200 import binding
    return binding


def test_every_declared_symbol_is_exported_and_bound(dense):
    header = open(os.path.join(ROOT, "include", "falqon_dense.h")).read()
    declared = set(re.findall(r"^(?:int|size_t) (falqon_[a-z_]+)\s*\(", header, flags=re.M))
    assert declared == set(dense.DENSE_EXPORTS)
    for name in declared:
        assert hasattr(dense.lib, name), name


def test_the_header_is_plain_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text('#include "falqon_dense.h"\nint main(void) { falqon_ortho o; falqon_blocking b = FALQON_TILE; (void)o; (void)b; return 0; }\n')
    for cmd in (["gcc", "-std=c99", "-pedantic"], ["g++", "-std=c++11", "-x", "c++"]):
        subprocess.run([*cmd, "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)], check=True)


def test_struct_layout_and_constants_match_the_header(dense, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    fields = [f for f, *_ in dense.falqon_ortho._fields_]
    lines = ['printf("%zu\\n", sizeof(falqon_ortho));'] + [f'printf("%zu\\n", offsetof(falqon_ortho, {f}));' for f in fields]
    lines += [f'printf("%zu\\n", (size_t){c});' for c in ("FALQON_BLOCK", "FALQON_ORTHO_MAX_STEPS", "FALQON_ALONG_ROW", "FALQON_ALONG_COL", "FALQON_TILE")]
    src.write_text('#include <stdio.h>\n#include "falqon_dense.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [C.sizeof(dense.falqon_ortho)] + [getattr(dense.falqon_ortho, f).offset for f in fields]
    want += [dense.BLOCK, dense.ORTHO_MAX_STEPS, dense.ALONG["row"], dense.ALONG["col"], dense.ALONG["tile"]]
    assert got == want


def test_quantizer_refusals(dense, fq):
    inv, lib = fq.ERR_INVALID_ARG, dense.lib
    ok = [FAKE, 0, 4, 8, 8, 0, 0, 2 * FAKE, 3 * FAKE, None]

    def refused(**at):
        args = list(ok)
        for k, v in at.items():
            args[int(k[1:])] = v
        return lib.falqon_block_quantize(*args) == inv

    assert refused(_0=None) and refused(_7=None) and refused(_8=None)
    assert refused(_1=2) and refused(_1=-1)                            # dtype
    assert refused(_2=0) and refused(_3=0) and refused(_2=-4)
    assert refused(_4=7) and refused(_4=(1 << 42) + 1)                 # row pitch
    assert refused(_5=2) and refused(_6=3) and refused(_6=-1)          # format, blocking
    assert refused(_2=(1 << 30) + 1) and refused(_2=1 << 30, _3=1 << 13, _4=1 << 13)       # sizes
    assert refused(_0=FAKE + 1) and refused(_0=FAKE + 2, _1=1)         # alignment to the type
    assert refused(_7=FAKE)                                            # in place
    both = [FAKE, 0, 4, 8, 8, 0, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE, None]
    for k in (0, 6, 7, 8, 9):
        assert lib.falqon_block_quantize_both(*(both[:k] + [None] + both[k + 1:])) == inv
    assert lib.falqon_block_quantize_both(*(both[:8] + [2 * FAKE] + both[9:])) == inv       # one buffer for both codes
    assert lib.falqon_block_quantize_both(*(both[:6] + [FAKE] + both[7:])) == inv
    back = [FAKE, FAKE, 0, 0, 4, 8, FAKE, 0, None]
    for k, v in ((0, None), (1, None), (6, None), (2, 2), (3, 3), (4, 0), (5, 0), (7, 2), (6, FAKE + 1)):
        assert lib.falqon_block_dequantize(*(back[:k] + [v] + back[k + 1:])) == inv


@pytest.mark.parametrize("call", ["falqon_block_forward", "falqon_block_input_grad", "falqon_block_weight_grad"])
def test_product_refusals(dense, fq, call):
    f = getattr(dense.lib, call)
    ok = [FAKE, FAKE, 0, FAKE, FAKE, 0, 64, 128, 256, FAKE, 0, None]
    for k, v in ((0, None), (1, None), (3, None), (4, None), (9, None), (2, 2), (5, -1), (10, 2), (6, 0), (6, -1), (6, (1 << 30) + 1), (7, 8), (7, 100), (7, 0),
                 (8, 24), (8, 0), (0, FAKE + 8), (3, FAKE + 8), (9, FAKE + 4)):
        assert f(*(ok[:k] + [v] + ok[k + 1:])) == fq.ERR_INVALID_ARG, (k, v)
    huge = 1 << 30          # more tiles than an int counts
    assert f(*(ok[:6] + [huge, huge, huge] + ok[9:])) == fq.ERR_INVALID_ARG


def test_linear_refusals_and_scratch(dense, fq):
    lib = dense.lib
    for T, m in ((1, 11008), (2, 11008), (4, 4096)):
        assert lib.falqon_block_linear_scratch_bytes(T, 4096, m) == 0           # one launch, no scratch
    assert lib.falqon_block_linear_scratch_bytes(5, 4096, 11008) == 5 * 4096 + 160
    assert lib.falqon_block_linear_scratch_bytes(100, 2064, 1040) == 100 * 2064 + 1712
    for bad in ((0, 128, 128), (1, 120, 128), (1, 128, 100), (-1, 128, 128), ((1 << 30) + 1, 128, 128)):
        assert lib.falqon_block_linear_scratch_bytes(*bad) == 0
    ok = [FAKE, 0, FAKE, FAKE, 0, 64, 128, 256, FAKE, 0, FAKE, 1 << 30, None]
    for k, v in ((0, None), (1, 2), (2, None), (3, None), (4, 3), (5, 0), (6, 100), (7, 8), (8, None), (9, 2), (0, FAKE + 8), (2, FAKE + 8), (8, FAKE + 8)):
        assert lib.falqon_block_linear(*(ok[:k] + [v] + ok[k + 1:])) == fq.ERR_INVALID_ARG, (k, v)
    for k, v in ((10, None), (10, FAKE + 8), (11, 64 * 128 + 63)):
        assert lib.falqon_block_linear(*(ok[:k] + [v] + ok[k + 1:])) == fq.ERR_WORKSPACE, (k, v)


def plan(dense, **kw):
    a = dict(batch=1, rows=64, cols=256, dtype=0, out_dtype=0, steps=5, eps=1e-7, scale=1.0, coefficients=None)
    a.update(kw)
    return dense.falqon_ortho(*a.values())


def test_orthogonalize_sizes_and_refusals(dense, fq):
    lib = dense.lib
    size = lambda **kw: lib.falqon_orthogonalize_scratch_bytes(C.byref(plan(dense, **kw)))  # noqa: E731
    assert size() > 0 and size(rows=32768, cols=32768) > 32768 * 32768 * 8
    for kw in (dict(batch=0), dict(batch=65536), dict(rows=0), dict(rows=32769), dict(cols=0), dict(cols=32769), dict(batch=1024, rows=32768, cols=32768), dict(dtype=2),
               dict(out_dtype=-1), dict(steps=0), dict(steps=33)):
        assert size(**kw) == 0, kw
        assert lib.falqon_orthogonalize(C.byref(plan(dense, **kw)), FAKE, FAKE, FAKE, 1 << 40, None) == fq.ERR_INVALID_ARG
    assert lib.falqon_orthogonalize_scratch_bytes(None) == 0
    go = lambda p, g=FAKE, out=2 * FAKE, ws=FAKE, n=1 << 40: lib.falqon_orthogonalize(C.byref(p), g, out, ws, n, None)  # noqa: E731
    assert go(plan(dense), g=None) == fq.ERR_INVALID_ARG and go(plan(dense), out=None) == fq.ERR_INVALID_ARG
    assert go(plan(dense), g=FAKE + 1) == fq.ERR_INVALID_ARG and go(plan(dense, out_dtype=1), out=FAKE + 2) == fq.ERR_INVALID_ARG
    assert go(plan(dense, out_dtype=1), out=FAKE) == fq.ERR_INVALID_ARG                    # in place with another type
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert go(plan(dense, **kw)) == fq.ERR_INVALID_ARG
    assert go(plan(dense), ws=None) == fq.ERR_WORKSPACE and go(plan(dense), ws=FAKE + 8) == fq.ERR_WORKSPACE
    assert go(plan(dense), n=size() - 1) == fq.ERR_WORKSPACE


@pytest.mark.parametrize("table,fits", [([(8.0, 0.0, 0.0)], False), ([(7.8, 0.0, 0.0)], True), ([(2.5, 0.0, 0.0)] * 2, True), ([(3.0, 0.0, 0.0)] * 2, False),
                                        ([(1.5, -0.5, 0.0)] * 32, True), ([(0.0, 9.0, 0.0)], False), ([(0.0, 0.0, -8.0)], False),
                                        ([(0.0, 30.0, -30.0)], True), ([(0.0, 33.0, -33.0)], False), ([(float("nan"), 0.0, 0.0)], False)])
def test_coefficients_are_held_to_the_range(dense, fq, table, fits):
    """A polynomial whose iterates could leave the range that they are held in is refused before the scratch is looked at (too small here).
    30 (x - x^2) is at most 7.5, 33 (x - x^2) 8.25."""
    flat = (C.c_float * (3 * len(table)))(*(v for c in table for v in c))
    p = plan(dense, steps=len(table), coefficients=flat)
    assert dense.lib.falqon_orthogonalize(C.byref(p), FAKE, 2 * FAKE, FAKE, 1, None) == (fq.ERR_WORKSPACE if fits else fq.ERR_INVALID_ARG)


def test_python_refusals(dense):
    """Checks that come before any tensor has to lie on a device."""
    x = torch.zeros((4, 32))
    for bad in (x[0], x[:0], x.T):
        with pytest.raises(ValueError):
            dense.block_quantize(bad)
    for kw in (dict(along="diagonal"), dict(fmt="e3m4")):
        with pytest.raises(ValueError):
            dense.block_quantize(x, **kw)
    codes = torch.zeros((4, 32), dtype=torch.float8_e4m3fn)
    row, tile = dense.Blocks(codes, torch.zeros((4, 1), dtype=torch.uint8), "row"), dense.Blocks(codes, torch.zeros((1, 1), dtype=torch.uint8), "tile")
    wide = dense.Blocks(torch.zeros((16, 32), dtype=torch.float8_e4m3fn), torch.zeros((1, 1), dtype=torch.uint8), "tile")
    for call in (lambda: dense.block_forward(row, row), lambda: dense.block_forward(tile, wide), lambda: dense.block_forward(row, tile),
                 lambda: dense.block_forward(row._replace(scales=torch.zeros((4, 2), dtype=torch.uint8)), wide),
                 lambda: dense.block_forward(row._replace(codes=codes.float()), wide), lambda: dense.block_input_grad(row, wide),
                 lambda: dense.block_weight_grad(row, row), lambda: dense.block_forward(x[:, :16].contiguous(), wide), lambda: dense.block_forward(x.T, wide),
                 lambda: dense.block_dequantize(row._replace(scales=row.scales.int())), lambda: dense.orthogonalize(x[0]), lambda: dense.orthogonalize(x, steps=0),
                 lambda: dense.orthogonalize(x, coefficients=[(1.0, 2.0)])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        dense.orthogonalize(x, dtype=torch.float16)
