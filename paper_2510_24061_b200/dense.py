"""A linear layer held, multiplied and updated in 8 bits by blocks: the calls of include/falqon_dense.h on torch tensors.

* ``block_quantize`` / ``block_quantize_both`` / ``block_dequantize``: codes with a power-of-two scale for each block of 128 values;
* ``block_forward`` / ``block_input_grad`` / ``block_weight_grad``: the three products of a layer held so; ``block_forward`` also takes
  unquantized tokens, which is the form for serving;
* ``orthogonalize``: an update orthogonalised by Newton-Schulz products, as the Muon optimizer takes it.

Argument checks and marshalling only, like ``training``; the arithmetic runs in the library's kernels, on the current stream.  These are not
autograd functions: results never require a gradient, and gradients are asked for by their own calls.
Tensors are on the current device, bf16 or fp32; codes are torch.float8_e4m3fn or torch.float8_e5m2.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence, Tuple, Union

import torch

from . import binding as fq
from .training import _dtype, _need, _new, _on_device, _ptr

lib = fq.lib
_p, _f, _i, _i64, _sz = C.c_void_p, C.c_float, C.c_int, C.c_int64, C.c_size_t


class falqon_ortho(C.Structure):
    _fields_ = [("batch", _i64), ("rows", _i64), ("cols", _i64), ("dtype", C.c_int32), ("out_dtype", C.c_int32), ("steps", C.c_int32),
                ("eps", _f), ("scale", _f), ("coefficients", C.POINTER(_f))]


_ortho_p = C.POINTER(falqon_ortho)
_SIGNATURES = {
    "falqon_block_quantize": (_i, [_p, _i, _i64, _i64, _i64, _i, _i, _p, _p, _p]),
    "falqon_block_quantize_both": (_i, [_p, _i, _i64, _i64, _i64, _i, _p, _p, _p, _p, _p]),
    "falqon_block_dequantize": (_i, [_p, _p, _i, _i, _i64, _i64, _p, _i, _p]),
    "falqon_block_forward": (_i, [_p, _p, _i, _p, _p, _i, _i64, _i64, _i64, _p, _i, _p]),
    "falqon_block_input_grad": (_i, [_p, _p, _i, _p, _p, _i, _i64, _i64, _i64, _p, _i, _p]),
    "falqon_block_weight_grad": (_i, [_p, _p, _i, _p, _p, _i, _i64, _i64, _i64, _p, _i, _p]),
    "falqon_block_linear_scratch_bytes": (_sz, [_i64, _i64, _i64]),
    "falqon_block_linear": (_i, [_p, _i, _p, _p, _i, _i64, _i64, _i64, _p, _i, _p, _sz, _p]),
    "falqon_orthogonalize_scratch_bytes": (_sz, [_ortho_p]),
    "falqon_orthogonalize": (_i, [_ortho_p, _p, _p, _p, _sz, _p]),
}
DENSE_EXPORTS = list(_SIGNATURES)
for _name, (_res, _args) in _SIGNATURES.items():
    getattr(lib, _name).restype = _res
    getattr(lib, _name).argtypes = _args

BLOCK = 128
ORTHO_MAX_STEPS = 32
ALONG = {"row": 0, "col": 1, "tile": 2}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_FMT_CODE = {torch.float8_e4m3fn: fq.E4M3, torch.float8_e5m2: fq.E5M2}


class Blocks(NamedTuple):
    """A [rows, cols] tensor in 8 bits: ``codes`` (torch.float8_e4m3fn or float8_e5m2) and ``scales`` uint8, where a byte e stands for
    2^(e - 127) and serves a block: ``along`` "row" 128 values of a row, scales [rows, ceil(cols / 128)]; "col" 128 values of a column,
    scales [ceil(rows / 128), cols]; "tile" 128 x 128 values, scales [ceil(rows / 128), ceil(cols / 128)]."""
    codes: torch.Tensor
    scales: torch.Tensor
    along: str


def _scale_shape(rows: int, cols: int, along: str) -> Tuple[int, int]:
    return (rows if along == "row" else -(-rows // BLOCK), cols if along == "col" else -(-cols // BLOCK))


def _blocks(q: Blocks, along: Union[str, Tuple[str, ...]], name: str):
    codes, scales, of = q
    if of not in along or codes.dtype not in _FMT_CODE or codes.dim() != 2 or not codes.is_contiguous() or codes.numel() == 0:
        raise ValueError(f"{name} must be Blocks along {along} with contiguous, non-empty [rows, cols] codes")
    shape = _scale_shape(*codes.shape, of)
    if scales.dtype != torch.uint8 or scales.shape != shape or not scales.is_contiguous():
        raise ValueError(f"{name}.scales must be a contiguous uint8 tensor of shape {shape}")


def _values(x: torch.Tensor, name: str):
    """(rows, cols, row pitch in values) of a matrix of consecutive values in a row."""
    if x.dim() == 2:
        (rows, cols), (pitch, step) = x.shape, x.stride()
        if rows == 1:
            pitch = cols
        if rows > 0 and cols > 0 and (step == 1 or cols == 1) and pitch >= cols:
            return rows, cols, pitch
    raise ValueError(f"{name} must be a non-empty [rows, cols] tensor of consecutive values")


def _format(fmt: str) -> torch.dtype:
    if fmt not in FORMATS:
        raise ValueError(f"fmt must be one of {sorted(FORMATS)}")
    return FORMATS[fmt]


def _new_blocks(rows: int, cols: int, along: str, codes: torch.dtype, device) -> Blocks:
    return Blocks(_new(rows, cols, dtype=codes, device=device), _new(*_scale_shape(rows, cols, along), dtype=torch.uint8, device=device), along)


def _result(out: Optional[torch.Tensor], rows: int, cols: int, dtype: torch.dtype, device, name: str) -> torch.Tensor:
    if out is None:
        return _new(rows, cols, dtype=dtype, device=device)
    if out.shape != (rows, cols) or out.dtype != dtype or not out.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {(rows, cols)}")
    return out


# ---------------------------------------------------------------------------------------------------------------- codes
def block_quantize(x: torch.Tensor, along: str = "row", fmt: str = "e4m3", out: Optional[Blocks] = None) -> Blocks:
    """falqon_block_quantize: x [rows, cols] (a row pitch is allowed) in 8 bits, a scale for each block of 128 values ``along`` a
    "row", a "col"umn, or for each 128 x 128 "tile".  fmt "e4m3" or "e5m2"."""
    if along not in ALONG:
        raise ValueError(f"along must be one of {sorted(ALONG)}")
    codes = _format(fmt)
    rows, cols, ld = _values(x, "x")
    if out is None:
        stream = _on_device(x)
        out = _new_blocks(rows, cols, along, codes, x.device)
    else:
        _blocks(out, (along,), "out")
        _need(out.codes.shape == x.shape and out.codes.dtype == codes, "out must hold codes like x in fmt")
        stream = _on_device(x, out.codes, out.scales)
    fq._check("falqon_block_quantize", lib.falqon_block_quantize(x.data_ptr(), _dtype(x), rows, cols, ld, _FMT_CODE[codes], ALONG[along],
                                                                 out.codes.data_ptr(), out.scales.data_ptr(), stream))
    return out


def block_quantize_both(x: torch.Tensor, fmt: str = "e4m3") -> Tuple[Blocks, Blocks]:
    """falqon_block_quantize_both: (along "row", along "col") from one read of x: what a training step needs of a layer's input and of
    its output's gradient."""
    codes = _format(fmt)
    rows, cols, ld = _values(x, "x")
    stream, device = _on_device(x), x.device
    row, col = _new_blocks(rows, cols, "row", codes, device), _new_blocks(rows, cols, "col", codes, device)
    fq._check("falqon_block_quantize_both",
              lib.falqon_block_quantize_both(x.data_ptr(), _dtype(x), rows, cols, ld, _FMT_CODE[codes], row.codes.data_ptr(), row.scales.data_ptr(),
                                             col.codes.data_ptr(), col.scales.data_ptr(), stream))
    return row, col


def block_dequantize(q: Blocks, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """falqon_block_dequantize: the values that codes stand for."""
    _blocks(q, tuple(ALONG), "q")
    stream = _on_device(q.codes, q.scales, out)
    out = _result(out, *q.codes.shape, dtype, q.codes.device, "out")
    fq._check("falqon_block_dequantize", lib.falqon_block_dequantize(q.codes.data_ptr(), q.scales.data_ptr(), _FMT_CODE[q.codes.dtype], ALONG[q.along],
                                                                     *q.codes.shape, out.data_ptr(), _dtype(out), stream))
    return out


# ---------------------------------------------------------------------------------------------------------------- products
def _layer(n: int, m: int):
    _need(n % 16 == 0 and m % 16 == 0, "a layer's input and output widths must be multiples of 16")


def block_forward(x: Union[Blocks, torch.Tensor], w: Blocks, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                  scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [T, m] = x w^T.  w [m, n]: Blocks by "tile"; x [T, n]: Blocks along "row" (falqon_block_forward), or a contiguous bf16 or fp32
    tensor, quantized to E4M3 along "row" on the way (falqon_block_linear: few tokens take one launch)."""
    _blocks(w, ("tile",), "w")
    m, n = w.codes.shape
    _layer(n, m)
    if isinstance(x, Blocks):
        _blocks(x, ("row",), "x")
        T = x.codes.shape[0]
        _need(x.codes.shape[1] == n, "x and w have different input widths")
        stream = _on_device(x.codes, x.scales, w.codes, w.scales, out)
        out = _result(out, T, m, dtype, w.codes.device, "out")
        fq._check("falqon_block_forward",
                  lib.falqon_block_forward(x.codes.data_ptr(), x.scales.data_ptr(), _FMT_CODE[x.codes.dtype], w.codes.data_ptr(), w.scales.data_ptr(),
                                           _FMT_CODE[w.codes.dtype], T, n, m, out.data_ptr(), _dtype(out), stream))
        return out
    _need(x.dim() == 2 and x.is_contiguous() and x.numel() > 0, "x must be a contiguous, non-empty [tokens, n] tensor or Blocks")
    T = x.shape[0]
    _need(x.shape[1] == n, "x and w have different input widths")
    stream = _on_device(x, w.codes, w.scales, out, scratch)
    out = _result(out, T, m, dtype, w.codes.device, "out")
    size = lib.falqon_block_linear_scratch_bytes(T, n, m)
    if scratch is None and size:
        scratch = _new(size, dtype=torch.uint8, device=x.device)
    fq._check("falqon_block_linear",
              lib.falqon_block_linear(x.data_ptr(), _dtype(x), w.codes.data_ptr(), w.scales.data_ptr(), _FMT_CODE[w.codes.dtype], T, n, m,
                                      out.data_ptr(), _dtype(out), _ptr(scratch), scratch.numel() * scratch.element_size() if scratch is not None else 0,
                                      stream))
    return out


def block_input_grad(dy: Blocks, w: Blocks, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """falqon_block_input_grad: dx [T, n] = dy w.  dy [T, m]: Blocks along "row"; w [m, n]: Blocks by "tile", as in the forward."""
    _blocks(dy, ("row",), "dy")
    _blocks(w, ("tile",), "w")
    m, n = w.codes.shape
    _layer(n, m)
    T = dy.codes.shape[0]
    _need(dy.codes.shape[1] == m, "dy and w have different output widths")
    stream = _on_device(dy.codes, dy.scales, w.codes, w.scales, out)
    out = _result(out, T, n, dtype, w.codes.device, "out")
    fq._check("falqon_block_input_grad",
              lib.falqon_block_input_grad(dy.codes.data_ptr(), dy.scales.data_ptr(), _FMT_CODE[dy.codes.dtype], w.codes.data_ptr(), w.scales.data_ptr(),
                                          _FMT_CODE[w.codes.dtype], T, n, m, out.data_ptr(), _dtype(out), stream))
    return out


def block_weight_grad(dy: Blocks, x: Blocks, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """falqon_block_weight_grad: dw [m, n] = dy^T x.  dy [T, m] and x [T, n]: Blocks along "col" (the contraction is over tokens)."""
    _blocks(dy, ("col",), "dy")
    _blocks(x, ("col",), "x")
    T, m = dy.codes.shape
    n = x.codes.shape[1]
    _layer(n, m)
    _need(x.codes.shape[0] == T, "dy and x have different numbers of tokens")
    stream = _on_device(dy.codes, dy.scales, x.codes, x.scales, out)
    out = _result(out, m, n, dtype, x.codes.device, "out")
    fq._check("falqon_block_weight_grad",
              lib.falqon_block_weight_grad(dy.codes.data_ptr(), dy.scales.data_ptr(), _FMT_CODE[dy.codes.dtype], x.codes.data_ptr(), x.scales.data_ptr(),
                                           _FMT_CODE[x.codes.dtype], T, n, m, out.data_ptr(), _dtype(out), stream))
    return out


# ---------------------------------------------------------------------------------------------------------------- the optimizer's update
def orthogonalize(g: torch.Tensor, steps: int = 5, coefficients: Optional[Sequence[Sequence[float]]] = None, eps: float = 1e-7, scale: float = 1.0,
                  dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None) -> torch.Tensor:
    """falqon_orthogonalize: scale * X after ``steps`` of X <- a X + (b G + c G G) X, G = X X^T, from X = g / (|g|_F + eps).
    g: contiguous [rows, cols] or [batch, rows, cols] (each matrix for itself), bf16 or fp32; the result is of its type or ``dtype``: bf16
    results are made of fp16 products, fp32 ones of three such products each.  coefficients: (a, b, c) of each step (steps is then their
    number), None: the Muon optimizer's 3.4445, -4.7750, 2.0315.  scratch: falqon_orthogonalize_scratch_bytes, allocated if None.  out may be g."""
    _need(g.dim() in (2, 3) and g.is_contiguous() and g.numel() > 0, "g must be a contiguous, non-empty [rows, cols] or [batch, rows, cols] tensor")
    dtype = (out.dtype if out is not None else g.dtype) if dtype is None else dtype
    if out is not None and (out.shape != g.shape or out.dtype != dtype or not out.is_contiguous()):
        raise ValueError(f"out must be a contiguous {dtype} tensor of shape {tuple(g.shape)}")
    table = None
    if coefficients is not None:
        _need(all(len(c) == 3 for c in coefficients), "coefficients are (a, b, c) of each step")
        steps = len(coefficients)
        table = (_f * (3 * steps))(*(v for c in coefficients for v in c))
    if not 1 <= steps <= ORTHO_MAX_STEPS:
        raise ValueError(f"steps must be 1 to {ORTHO_MAX_STEPS}")
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype}")
    rows, cols = g.shape[-2:]
    plan = falqon_ortho(g.shape[0] if g.dim() == 3 else 1, rows, cols, _dtype(g), fq.BF16 if dtype == torch.bfloat16 else fq.F32, steps, eps, scale, table)
    stream = _on_device(g, out, scratch)
    out = torch.empty(g.shape, dtype=dtype, device=g.device) if out is None else out
    size = lib.falqon_orthogonalize_scratch_bytes(C.byref(plan))
    if size == 0:
        raise fq.FalqonError("falqon_orthogonalize_scratch_bytes", fq.ERR_INVALID_ARG)
    if scratch is None:
        scratch = _new(size, dtype=torch.uint8, device=g.device)
    fq._check("falqon_orthogonalize",
              lib.falqon_orthogonalize(C.byref(plan), g.data_ptr(), out.data_ptr(), scratch.data_ptr(), scratch.numel() * scratch.element_size(), stream))
    return out
