"""What a fine-tuning step runs between and behind the melded layers: the calls of include/falqon_train.h on torch tensors.

* ``block_norm_forward`` / ``block_norm_backward``: the norms after and before a block, with its gate and the residual scale;
* ``checkpoint_save`` / ``checkpoint_load``, ``gate_forward`` / ``gate_backward``: activations kept in 8 bits for the backward;
* ``preference_forward`` / ``preference_backward``, ``sequence_logprob``: the loss of paired sequences.

Argument checks and marshalling only, like ``binding``; the arithmetic runs in the library's kernels, on the current stream.
Tensors are contiguous (logits may have a row pitch), on the current device, bf16 or fp32.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence, Union

import torch

from . import binding as fq

lib = fq.lib
_p, _f, _i, _i64, _sz = C.c_void_p, C.c_float, C.c_int, C.c_int64, C.c_size_t


class falqon_block_norm(C.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("rows_per_gate", _i64), ("dtype", C.c_int32), ("gain_dtype", C.c_int32),
                ("flags", C.c_int32), ("res_scale", _f), ("gain_offset", _f), ("eps", _f), ("post_gain", _p), ("pre_gain", _p),
                ("gate", _p)]


class falqon_preference(C.Structure):
    _fields_ = [("rows", _i64), ("vocab", _i64), ("ld", _i64), ("pairs", _i64), ("dtype", C.c_int32), ("kind", C.c_int32),
                ("flags", C.c_int32), ("beta", _f), ("margin", _f), ("label_smoothing", _f), ("nll_weight", _f)]


_norm_p, _pref_p = C.POINTER(falqon_block_norm), C.POINTER(falqon_preference)
_SIGNATURES = {
    "falqon_checkpoint_save": (_i, [_p, _i, _i64, _i64, _p, _p, _p]),
    "falqon_checkpoint_load": (_i, [_p, _p, _i64, _i64, _p, _i, _p]),
    "falqon_gate_forward": (_i, [_p, _p, _i, _i64, _i64] + [_p] * 7),
    "falqon_gate_backward": (_i, [_p] * 5 + [_i, _i64, _i64] + [_p] * 5),
    "falqon_block_norm_forward": (_i, [_norm_p] + [_p] * 12),
    "falqon_block_norm_scratch_bytes": (_sz, [_norm_p]),
    "falqon_block_norm_backward": (_i, [_norm_p] + [_p] * 17 + [_sz, _p]),
    "falqon_preference_scratch_bytes": (_sz, [_i64, _i64, _i]),
    "falqon_sequence_logprob": (_i, [_p, _i, _i64, _i64, _i64, _p, _p, _i64, _i, _p, _p, _p, _sz, _p]),
    "falqon_preference_forward": (_i, [_pref_p] + [_p] * 11 + [_sz, _p]),
    "falqon_preference_backward": (_i, [_pref_p] + [_p] * 6 + [_i64, _p, _p]),
}
TRAIN_EXPORTS = list(_SIGNATURES)
for _name, (_res, _args) in _SIGNATURES.items():
    getattr(lib, _name).restype = _res
    getattr(lib, _name).argtypes = _args

NORM_POST, NORM_PRE, NORM_MAX_COLS, NORM_MAX_ROWS = 1, 2, 16384, (1 << 31) - 1024
CHECKPOINT_BLOCK = 32
PREFERENCE_KINDS = {"sigmoid": 0, "hinge": 1, "ipo": 2}
_DTYPES = {torch.bfloat16: fq.BF16, torch.float32: fq.F32}


def _new(*shape: int, dtype: torch.dtype, device) -> torch.Tensor:
    """An uninitialised contiguous tensor on the current device.  The four outputs of a one-row norm take 5.8 us by torch.empty and
    torch.empty_like, of 17 us for the whole call, and 3.8 us by the allocator entry that torch's generated code uses, where torch has
    it: it skips the parsing of a device and its guard."""
    if _empty_cuda is None:
        return torch.empty(shape, dtype=dtype, device=device)
    stride = (shape[1], 1) if len(shape) == 2 else (1,) * len(shape)
    return _empty_cuda(shape, stride, dtype)


def _new_checkpoint(x: torch.Tensor) -> "Checkpoint":
    rows, cols = x.shape
    return Checkpoint(_new(rows, cols, dtype=torch.uint8, device=x.device),
                      _new(rows, (cols + CHECKPOINT_BLOCK - 1) // CHECKPOINT_BLOCK, dtype=torch.uint8, device=x.device))


_empty_cuda = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _dtype(t: torch.Tensor) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def _on_device(*tensors) -> int:
    """The current stream's handle, the tensors being checked to lie on the current device.  (A third of a small call's time was the
    stream object that torch.cuda.current_stream() makes: the handle alone is enough here.)"""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor on {t.device} where the current device is cuda:{dev}")
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream


def _like(t: Optional[torch.Tensor], ref: torch.Tensor, name: str):
    if t is not None and (t.dtype != ref.dtype or t.shape != ref.shape or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {ref.dtype} tensor of shape {tuple(ref.shape)}")


def _vector(t: Optional[torch.Tensor], n: int, dtype: torch.dtype, name: str):
    if t is not None and (t.dtype != dtype or t.numel() != n or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} entries")


def _matrix(t: torch.Tensor, name: str):
    if t.dim() != 2 or not t.is_contiguous() or t.numel() == 0:
        raise ValueError(f"{name} must be a contiguous, non-empty [rows, cols] tensor")


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---------------------------------------------------------------------------------------------------------------- checkpoints
class Checkpoint(NamedTuple):
    """An activation in 8 bits: E4M3 ``codes`` uint8 [rows, cols] and ``scales`` uint8 [rows, ceil(cols / 32)], where a byte e
    stands for 2^(e - 127) and serves 32 consecutive values of its row."""
    codes: torch.Tensor
    scales: torch.Tensor

    @staticmethod
    def empty(rows: int, cols: int, device) -> "Checkpoint":
        blocks = -(-cols // CHECKPOINT_BLOCK)
        return Checkpoint(torch.empty_strided((rows, cols), (cols, 1), dtype=torch.uint8, device=device),
                          torch.empty_strided((rows, blocks), (blocks, 1), dtype=torch.uint8, device=device))


def _checkpoint(ck: Checkpoint, shape, name: str):
    rows, cols = shape
    codes, scales = ck
    if (codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.shape != shape
            or scales.shape != (rows, -(-cols // CHECKPOINT_BLOCK)) or not codes.is_contiguous() or not scales.is_contiguous()):
        raise ValueError(f"{name} must be a Checkpoint of a [{rows}, {cols}] tensor")


def checkpoint_save(x: torch.Tensor, out: Optional[Checkpoint] = None) -> Checkpoint:
    """falqon_checkpoint_save: x [rows, cols] in 8 bits."""
    _matrix(x, "x")
    stream = _on_device(x)
    out = _new_checkpoint(x) if out is None else out
    _checkpoint(out, x.shape, "out")
    _on_device(*out)
    fq._check("falqon_checkpoint_save", lib.falqon_checkpoint_save(x.data_ptr(), _dtype(x), *x.shape, out.codes.data_ptr(),
                                                                    out.scales.data_ptr(), stream))
    return out


def checkpoint_load(ck: Checkpoint, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """falqon_checkpoint_load: the values a checkpoint stands for."""
    _matrix(ck.codes, "ck.codes")
    _checkpoint(ck, ck.codes.shape, "ck")
    out = torch.empty(ck.codes.shape, dtype=dtype, device=ck.codes.device) if out is None else out
    _matrix(out, "out")
    _need(out.shape == ck.codes.shape, "out has another shape than the checkpoint")
    stream = _on_device(*ck, out)
    fq._check("falqon_checkpoint_load", lib.falqon_checkpoint_load(ck.codes.data_ptr(), ck.scales.data_ptr(), *out.shape,
                                                                    out.data_ptr(), _dtype(out), stream))
    return out


def gate_forward(g: torch.Tensor, u: torch.Tensor, save: bool = True, z: Optional[torch.Tensor] = None,
                 amax: Optional[torch.Tensor] = None):
    """falqon_gate_forward: z = silu(g) * u.  Returns (z, checkpoint of g, checkpoint of u), the latter two None without save.
    amax (fp32 [1], zero beforehand): raised to max |z|."""
    _matrix(g, "g")
    _like(u, g, "u")
    _like(z, g, "z")
    _vector(amax, 1, torch.float32, "amax")
    stream = _on_device(g, u, z, amax)
    z = _new(*g.shape, dtype=g.dtype, device=g.device) if z is None else z
    kg = ku = None
    ptrs = (None,) * 4
    if save:
        kg, ku = _new_checkpoint(g), _new_checkpoint(g)
        ptrs = (kg.codes.data_ptr(), kg.scales.data_ptr(), ku.codes.data_ptr(), ku.scales.data_ptr())
    fq._check("falqon_gate_forward", lib.falqon_gate_forward(g.data_ptr(), u.data_ptr(), _dtype(g), *g.shape, z.data_ptr(), *ptrs,
                                                              _ptr(amax), stream))
    return z, kg, ku


def gate_backward(g: Checkpoint, u: Checkpoint, dz: torch.Tensor, dg: Optional[torch.Tensor] = None,
                  du: Optional[torch.Tensor] = None, amax_dg: Optional[torch.Tensor] = None,
                  amax_du: Optional[torch.Tensor] = None):
    """falqon_gate_backward: (dg, du) from the checkpoints of g and u.  dg or du may be dz itself."""
    _matrix(dz, "dz")
    _checkpoint(g, dz.shape, "g")
    _checkpoint(u, dz.shape, "u")
    _like(dg, dz, "dg")
    _like(du, dz, "du")
    _vector(amax_dg, 1, torch.float32, "amax_dg")
    _vector(amax_du, 1, torch.float32, "amax_du")
    stream = _on_device(*g, *u, dz, dg, du, amax_dg, amax_du)
    dg = _new(*dz.shape, dtype=dz.dtype, device=dz.device) if dg is None else dg
    du = _new(*dz.shape, dtype=dz.dtype, device=dz.device) if du is None else du
    fq._check("falqon_gate_backward",
              lib.falqon_gate_backward(g.codes.data_ptr(), g.scales.data_ptr(), u.codes.data_ptr(), u.scales.data_ptr(), dz.data_ptr(),
                                       _dtype(dz), *dz.shape, dg.data_ptr(), du.data_ptr(), _ptr(amax_dg), _ptr(amax_du), stream))
    return dg, du


# ---------------------------------------------------------------------------------------------------------------- block norms
class BlockNormOut(NamedTuple):
    h_out: Optional[torch.Tensor]        # [rows, cols]
    x: Optional[torch.Tensor]            # [rows, cols], None without the norm before the next block
    inv_post: Optional[torch.Tensor]     # fp32 [rows]: what the backward needs of each norm
    inv_pre: Optional[torch.Tensor]
    saved_h: Optional[Checkpoint]        # with save
    saved_y: Optional[Checkpoint]


_GAINS = ("post_gain", "pre_gain", "gate")


class BlockNormGrad(NamedTuple):
    dh: Optional[torch.Tensor]
    dy: Optional[torch.Tensor]
    dpost_gain: Optional[torch.Tensor]   # fp32
    dpre_gain: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]


def _norm_plan(rows, cols, dtype, post, pre, post_gain, pre_gain, gate, rows_per_gate, res_scale, gain_offset, eps):
    gain = next((t for t in (post_gain, pre_gain, gate) if t is not None), None)
    gain_dtype = torch.float32 if gain is None else gain.dtype
    _need(post or post_gain is None, "post_gain without the norm after the block")
    _need(pre or pre_gain is None, "pre_gain without the norm before the next block")
    if post_gain is not None:
        _vector(post_gain, cols, gain_dtype, "post_gain")
    if pre_gain is not None:
        _vector(pre_gain, cols, gain_dtype, "pre_gain")
    rows_per_gate = rows if rows_per_gate is None else rows_per_gate
    _need(rows_per_gate >= 1, "rows_per_gate must be at least 1")
    if gate is not None:
        _vector(gate, -(-rows // rows_per_gate) * cols, gain_dtype, "gate")
    return falqon_block_norm(rows, cols, rows_per_gate, dtype, _DTYPES.get(gain_dtype, -1), (NORM_POST if post else 0) | (NORM_PRE if pre else 0),
                             res_scale, gain_offset, eps, _ptr(post_gain), _ptr(pre_gain), _ptr(gate))


def block_norm_forward(h: Optional[torch.Tensor], y: torch.Tensor, *, post: bool = True, pre: bool = True,
                       post_gain: Optional[torch.Tensor] = None, pre_gain: Optional[torch.Tensor] = None,
                       gate: Optional[torch.Tensor] = None, rows_per_gate: Optional[int] = None, res_scale: float = 1.0,
                       gain_offset: float = 0.0, eps: float = 1e-6, save: bool = False, h_out: Optional[torch.Tensor] = None,
                       x: Optional[torch.Tensor] = None, amax_x: Optional[torch.Tensor] = None, need_h_out: bool = True) -> BlockNormOut:
    """falqon_block_norm_forward.  y [rows, cols]: what the block gave; h: the residual stream before it (None: there is none).
        n = rmsnorm(y) * (gain_offset + post_gain)      (n = y without post)
        h_out = res_scale * h + gate * n                gate [ceil(rows / rows_per_gate), cols], one row per rows_per_gate rows
        x = rmsnorm(h_out) * (gain_offset + pre_gain)   (with pre)
    A gain or gate that is None is 1.  save: h and y are kept in 8 bits for the backward.  need_h_out False (with pre): only x is wanted,
    as before the head."""
    _matrix(y, "y")
    if not need_h_out:
        _need(pre and h_out is None, "a call without h_out is one with the norm before the next block and no h_out given")
    if h is not None:
        _like(h, y, "h")
    if h_out is not None:
        _like(h_out, y, "h_out")
    if x is not None:
        _like(x, y, "x")
    if amax_x is not None:
        _vector(amax_x, 1, torch.float32, "amax_x")
    rows, cols = y.shape
    plan = _norm_plan(rows, cols, _dtype(y), post, pre, post_gain, pre_gain, gate, rows_per_gate, res_scale, gain_offset, eps)
    stream = _on_device(h, y, h_out, x, amax_x, post_gain, pre_gain, gate)
    dtype, dev = y.dtype, y.device
    h_out = _new(rows, cols, dtype=dtype, device=dev) if h_out is None and need_h_out else h_out
    x = _new(rows, cols, dtype=dtype, device=dev) if x is None and pre else x
    inv_post = _new(rows, dtype=torch.float32, device=dev) if post else None
    inv_pre = _new(rows, dtype=torch.float32, device=dev) if pre else None
    kh = _new_checkpoint(y) if save and h is not None else None
    ky = _new_checkpoint(y) if save else None
    fq._check("falqon_block_norm_forward",
              lib.falqon_block_norm_forward(C.byref(plan), _ptr(h), y.data_ptr(), h_out.data_ptr() if h_out is not None else None, _ptr(x), _ptr(inv_post),
                                            _ptr(inv_pre),
                                            *((None, None) if kh is None else (kh.codes.data_ptr(), kh.scales.data_ptr())),
                                            *((None, None) if ky is None else (ky.codes.data_ptr(), ky.scales.data_ptr())),
                                            _ptr(amax_x), stream))
    return BlockNormOut(h_out, x if pre else None, inv_post, inv_pre, kh, ky)


def block_norm_backward(dx: Optional[torch.Tensor], dh_out: Optional[torch.Tensor], h: Union[torch.Tensor, Checkpoint, None],
                        y: Union[torch.Tensor, Checkpoint], inv_post: Optional[torch.Tensor], inv_pre: Optional[torch.Tensor], *,
                        post: bool = True, pre: bool = True, post_gain: Optional[torch.Tensor] = None,
                        pre_gain: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                        rows_per_gate: Optional[int] = None, res_scale: float = 1.0, gain_offset: float = 0.0, eps: float = 1e-6,
                        need_gains: Union[bool, Sequence[str]] = True, need_dy: bool = True, dh: Optional[torch.Tensor] = None,
                        dy: Optional[torch.Tensor] = None, scratch: Optional[torch.Tensor] = None, amax_dy: Optional[torch.Tensor] = None) -> BlockNormGrad:
    """falqon_block_norm_backward.  dx, dh_out: gradients of x (None without pre) and h_out (None: 0); h, y: the forward's inputs,
    as tensors or as its checkpoints; need_gains False: gains and gate are frozen and get no gradient, or the names of those that do
    ("post_gain", "pre_gain", "gate"); need_dy False: the block itself is frozen.  dh or dy may be dx or dh_out."""
    ref = dx if dx is not None else dh_out
    _need(ref is not None, "a backward needs dx or dh_out")
    _need(pre == (dx is not None), "dx goes with the norm before the next block")
    _matrix(ref, "dx")
    rows, cols = ref.shape
    for t, name in ((dh_out, "dh_out"), (dh, "dh"), (dy, "dy")):
        if t is not None:
            _like(t, ref, name)
    coded = isinstance(y, Checkpoint)
    _need(h is None or isinstance(h, Checkpoint) == coded, "h and y are saved in the same way")
    if coded:
        _checkpoint(y, ref.shape, "y")
        saved = [None, None, None, None, y.codes.data_ptr(), y.scales.data_ptr()]
        kept = y
        if h is not None:
            _checkpoint(h, ref.shape, "h")
            saved[1], saved[2] = h.codes.data_ptr(), h.scales.data_ptr()
            kept = (*y, *h)
    else:
        _like(y, ref, "y")
        if h is not None:
            _like(h, ref, "h")
        saved = [_ptr(h), None, None, y.data_ptr(), None, None]
        kept = (h, y)
    if post:
        _need(inv_post is not None, "inv_post of the forward is needed")
        _vector(inv_post, rows, torch.float32, "inv_post")
    if pre:
        _need(inv_pre is not None, "inv_pre of the forward is needed")
        _vector(inv_pre, rows, torch.float32, "inv_pre")
    if amax_dy is not None:
        _vector(amax_dy, 1, torch.float32, "amax_dy")
    if not need_dy:
        _need(dy is None and amax_dy is None, "dy or its absmax given where it is not wanted")
    of_post = of_pre = of_gate = need_gains is True
    if need_gains is not True and need_gains is not False:
        _need(not isinstance(need_gains, str) and set(need_gains) <= set(_GAINS), f"need_gains must be a bool or some of {_GAINS}")
        of_post, of_pre, of_gate = (name in need_gains for name in _GAINS)
    plan = _norm_plan(rows, cols, _dtype(ref), post, pre, post_gain, pre_gain, gate, rows_per_gate, res_scale, gain_offset, eps)
    stream = _on_device(dx, dh_out, inv_post, inv_pre, post_gain, pre_gain, gate, dh, dy, scratch, amax_dy, *kept)
    dev, dtype, f32 = ref.device, ref.dtype, torch.float32
    dh = _new(rows, cols, dtype=dtype, device=dev) if dh is None and h is not None else dh
    dy = _new(rows, cols, dtype=dtype, device=dev) if dy is None and need_dy else dy
    dpost = _new(cols, dtype=f32, device=dev) if of_post and post_gain is not None else None
    dpre = _new(cols, dtype=f32, device=dev) if of_pre and pre_gain is not None else None
    dgate = torch.empty(gate.shape, dtype=f32, device=dev) if of_gate and gate is not None else None
    size = 0
    if dpost is not None or dpre is not None or dgate is not None:
        size = lib.falqon_block_norm_scratch_bytes(C.byref(plan))
        if scratch is None:
            scratch = _new(size, dtype=torch.uint8, device=dev)
        size = scratch.numel() * scratch.element_size()
    fq._check("falqon_block_norm_backward",
              lib.falqon_block_norm_backward(C.byref(plan), _ptr(dx), _ptr(dh_out), *saved, _ptr(inv_post), _ptr(inv_pre), _ptr(dh),
                                             dy.data_ptr() if dy is not None else None,
                                             _ptr(dpost), _ptr(dpre), _ptr(dgate), _ptr(amax_dy), _ptr(scratch), size, stream))
    return BlockNormGrad(dh, dy, dpost, dpre, dgate)


# ---------------------------------------------------------------------------------------------------------------- preference loss
class PreferenceLoss(NamedTuple):
    """u = (seq_logp - ref)(chosen) - (seq_logp - ref)(rejected), D = beta * u - margin; kind "sigmoid": the negative log-sigmoid of
    D (with label_smoothing, mixed with that of -D), "hinge": max(0, 1 - D), "ipo": (u - margin - 1 / (2 beta))^2.  average: a
    sequence's log-probability is the mean over its counted rows.  nll_weight: plus so much of the chosen sequence's mean -logp."""
    kind: str = "sigmoid"
    beta: float = 0.1
    margin: float = 0.0
    label_smoothing: float = 0.0
    average: bool = False
    nll_weight: float = 0.0


class PreferenceOut(NamedTuple):
    loss: torch.Tensor                   # fp32, a scalar
    pair_loss: torch.Tensor              # fp32 [pairs]
    seq_logp: torch.Tensor               # fp32 [2 * pairs]
    logp: torch.Tensor                   # fp32 [rows]
    row_stats: Optional[torch.Tensor]    # fp32 [rows, 2], dlogp fp32 [rows]: for the backward
    dlogp: Optional[torch.Tensor]
    spec: PreferenceLoss


def _logits_ok(logits: torch.Tensor, name: str):
    if logits.dim() != 2 or logits.numel() == 0 or logits.stride(1) != 1 or (logits.shape[0] > 1 and logits.stride(0) < logits.shape[1]):
        raise ValueError(f"{name} must be a non-empty [rows, vocab] tensor of consecutive values")


def _pitch(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _preference(spec: PreferenceLoss, logits: torch.Tensor, pairs: int) -> falqon_preference:
    _need(spec.kind in PREFERENCE_KINDS, f"kind must be one of {sorted(PREFERENCE_KINDS)}")
    return falqon_preference(logits.shape[0], logits.shape[1], _pitch(logits), pairs, _dtype(logits), PREFERENCE_KINDS[spec.kind],
                             1 if spec.average else 0, spec.beta, spec.margin, spec.label_smoothing, spec.nll_weight)


def _scratch(logits: torch.Tensor, scratch: Optional[torch.Tensor]) -> torch.Tensor:
    if scratch is not None:
        return scratch
    size = lib.falqon_preference_scratch_bytes(logits.shape[0], logits.shape[1], _dtype(logits))
    if size == 0:
        raise fq.FalqonError("falqon_preference_scratch_bytes", fq.ERR_INVALID_ARG)
    return _new(size, dtype=torch.uint8, device=logits.device)


def sequence_logprob(logits: torch.Tensor, targets: torch.Tensor, cu_rows: torch.Tensor, average: bool = False,
                     scratch: Optional[torch.Tensor] = None):
    """falqon_sequence_logprob: (seq_logp [sequences], logp [rows]), fp32.  logits [rows, vocab] (a row pitch is allowed); targets int64
    [rows], negative where a row is not counted; cu_rows int64 [sequences + 1]: sequence i owns rows cu_rows[i] .. cu_rows[i + 1]."""
    _logits_ok(logits, "logits")
    rows, n = logits.shape[0], cu_rows.numel() - 1
    _need(n >= 1, "cu_rows must hold at least two entries")
    _vector(targets, rows, torch.int64, "targets")
    _vector(cu_rows, n + 1, torch.int64, "cu_rows")
    stream = _on_device(logits, targets, cu_rows, scratch)
    scratch = _scratch(logits, scratch)
    logp, seq = _new(rows, dtype=torch.float32, device=logits.device), _new(n, dtype=torch.float32, device=logits.device)
    fq._check("falqon_sequence_logprob",
              lib.falqon_sequence_logprob(logits.data_ptr(), _dtype(logits), rows, logits.shape[1], _pitch(logits), targets.data_ptr(),
                                          cu_rows.data_ptr(), n, int(average), logp.data_ptr(), seq.data_ptr(), scratch.data_ptr(),
                                          scratch.numel() * scratch.element_size(), stream))
    return seq, logp


def preference_forward(spec: PreferenceLoss, logits: torch.Tensor, targets: torch.Tensor, cu_rows: torch.Tensor,
                       ref_logp: Optional[torch.Tensor] = None, need_grad: bool = True,
                       scratch: Optional[torch.Tensor] = None) -> PreferenceOut:
    """falqon_preference_forward: the loss of packed sequences, pair p being sequences 2p (chosen) and 2p + 1 (rejected); arguments
    as in sequence_logprob.  ref_logp fp32 [2 * pairs]: the reference model's seq_logp (None: 0)."""
    _logits_ok(logits, "logits")
    rows, n = logits.shape[0], cu_rows.numel() - 1
    _need(n >= 2 and n % 2 == 0, "cu_rows must hold 2 * pairs + 1 entries")
    _vector(targets, rows, torch.int64, "targets")
    _vector(cu_rows, n + 1, torch.int64, "cu_rows")
    _vector(ref_logp, n, torch.float32, "ref_logp")
    plan = _preference(spec, logits, n // 2)
    stream = _on_device(logits, targets, cu_rows, ref_logp, scratch)
    scratch = _scratch(logits, scratch)
    f32, dev = torch.float32, logits.device
    loss, pair_loss, seq, logp = (_new(*shape, dtype=f32, device=dev) for shape in ((), (n // 2,), (n,), (rows,)))
    stats, dlogp = (_new(rows, 2, dtype=f32, device=dev), _new(rows, dtype=f32, device=dev)) if need_grad else (None, None)
    fq._check("falqon_preference_forward",
              lib.falqon_preference_forward(C.byref(plan), logits.data_ptr(), targets.data_ptr(), cu_rows.data_ptr(), _ptr(ref_logp),
                                            loss.data_ptr(), pair_loss.data_ptr(), seq.data_ptr(), logp.data_ptr(), _ptr(stats), _ptr(dlogp),
                                            scratch.data_ptr(), scratch.numel() * scratch.element_size(), stream))
    return PreferenceOut(loss, pair_loss, seq, logp, stats, dlogp, spec)


def preference_backward(logits: torch.Tensor, targets: torch.Tensor, out: PreferenceOut, dloss: Optional[torch.Tensor] = None,
                        dlogits: Optional[torch.Tensor] = None, amax: Optional[torch.Tensor] = None) -> torch.Tensor:
    """falqon_preference_backward: d loss / d logits times dloss (fp32 [1] on the device; None: 1).  dlogits may be logits itself."""
    _logits_ok(logits, "logits")
    _need(out.row_stats is not None, "the forward was called without need_grad")
    stream = _on_device(logits, targets, out.row_stats, out.dlogp, dloss, dlogits, amax)
    _vector(targets, logits.shape[0], torch.int64, "targets")
    _vector(out.dlogp, logits.shape[0], torch.float32, "out.dlogp")
    _vector(out.row_stats, 2 * logits.shape[0], torch.float32, "out.row_stats")
    _vector(dloss, 1, torch.float32, "dloss")
    _vector(amax, 1, torch.float32, "amax")
    if dlogits is None:
        dlogits = _new(*logits.shape, dtype=logits.dtype, device=logits.device)
    else:
        _logits_ok(dlogits, "dlogits")
        _need(dlogits.shape == logits.shape and dlogits.dtype == logits.dtype, "dlogits must be like logits")
    plan = _preference(out.spec, logits, out.pair_loss.numel())
    fq._check("falqon_preference_backward",
              lib.falqon_preference_backward(C.byref(plan), logits.data_ptr(), targets.data_ptr(), out.row_stats.data_ptr(),
                                             out.dlogp.data_ptr(), _ptr(dloss), dlogits.data_ptr(), _pitch(dlogits), _ptr(amax), stream))
    return dlogits
