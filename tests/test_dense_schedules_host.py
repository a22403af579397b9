"""Coefficients that change from step to step: published schedules of the polar factor's polynomials are taken (host side, no GPU)."""
import ctypes as C

import pytest

# Optimal odd quintics for singular values from 1e-3 to 1, each fitted to the range that the step before leaves, and the last for all further
# steps; to be divided by a safety factor's powers, since what rounding adds would leave the range at its upper end (a_k / f, b_k / f^3, c_k / f^5).
TIGHT = [(8.28721201814563, -23.595886519098837, 17.300387312530933), (4.107059111542203, -2.9478499167379106, 0.5448431082926601),
         (3.9486908534822946, -2.908902115962949, 0.5518191394370137), (3.3184196573706015, -2.488488024314874, 0.51004894012372),
         (2.300652019954817, -1.6689039845747493, 0.4188073119525673), (1.891301407787398, -1.2679958271945868, 0.37680408948524835),
         (1.8750014808534479, -1.2500016453999487, 0.3750001645474248), (1.875, -1.25, 0.375)]
SAFE = [(a / 1.01, b / 1.01 ** 3, c / 1.01 ** 5) for a, b, c in TIGHT]
# The same with a larger safety factor, in five steps.
FIVE = [(8.156554524902461, -22.48329292557795, 15.878769915207462), (4.042929935166739, -2.808917465908714, 0.5000178451051316),
        (3.8916678022926607, -2.772484153217685, 0.5060648178503393), (3.285753657755655, -2.3681294933425376, 0.46449024233002106),
        (2.3465413258596377, -1.7097828382687081, 0.42323551169305323)]


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import build
    build.build()
    from paper_2510_24061_b200 import dense
    return dense


def taken(dense, table, rows=256, cols=512, out_dtype=0):
    """Whether the table passes the checks, which come before that of the scratch (too small here)."""
    from paper_2510_24061_b200 import binding as fq
    flat = (C.c_float * (3 * len(table)))(*(v for c in table for v in c))
    p = dense.falqon_ortho(1, rows, cols, 0, out_dtype, len(table), 1e-7, 1.0, flat)
    rc = dense.lib.falqon_orthogonalize(C.byref(p), 0x10000, 0x20000, 0x10000, 1, None)
    assert rc in (fq.ERR_WORKSPACE, fq.ERR_INVALID_ARG)
    return rc == fq.ERR_WORKSPACE


@pytest.mark.parametrize("rows,cols", [(256, 512), (64, 900)])
@pytest.mark.parametrize("out_dtype", [0, 1])
def test_published_schedules_are_taken(dense, rows, cols, out_dtype):
    for steps in (1, 5, 8, 32):
        assert taken(dense, (SAFE + SAFE[-1:] * 24)[:steps], rows, cols, out_dtype), steps
    assert taken(dense, FIVE, rows, cols, out_dtype)
    # without the safety factor the iterates may leave the polynomials' range, and do so ever faster
    assert not taken(dense, TIGHT, rows, cols, out_dtype)
