"""Operators of a linear layer that is held, multiplied and updated in 8 bits by blocks, as cases that can be timed and checked:

* ``quant``: 8-bit codes with a power-of-two scale for each block of 128 values: of a row, of a column, or of a 128 x 128 tile;
* ``linear``: a few tokens through a layer whose weights are held so (serving), the tokens quantized on the way;
* ``prod``: the three products of training on such codes: forward, input gradient, weight gradient;
* ``ortho``: an update orthogonalised by Newton-Schulz products (the Muon optimizer's), single matrices and batches of them.

``run`` computes them in plain torch operations in 32 bits, or, where ``own`` is set, by the package's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP_EXPONENT = {"e4m3": 8, "e5m2": 15}      # the largest finite value is 1.75 * 2^this
QUINTIC = (3.4445, -4.7750, 2.0315)         # the Muon optimizer's polynomial, five times
STEPS, EPS = 5, 1e-7


# ---------------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a block's input in a training step of 4096 tokens: codes along the rows for the forward, along the columns for the weight gradient
        dict(name="quant both ways, 7B", op="quant", way="both", rows=4096, cols=4096, dtype="bf16", fmt="e4m3"),
        # the MLP's 32-bit weights after an optimizer step, a scale for each 128 x 128
        dict(name="quant tiles, 7B MLP, f32", op="quant", way="tile", rows=11008, cols=4096, dtype="f32", fmt="e4m3"),
        # a ragged gradient of a small model, blocks that end inside a row and a column
        dict(name="quant both ways, odd, f32", op="quant", way="both", rows=613, cols=1011, dtype="f32", fmt="e5m2"),
        # a single token through the MLP's first projection: decoding
        dict(name="linear, one token", op="linear", rows=1, n=4096, m=11008, dtype="bf16", out="bf16"),
        # a handful of sequences decoding together through a layer of odd sizes, blocks that end inside both
        dict(name="linear, 19 tokens, odd", op="linear", rows=19, n=2064, m=1040, dtype="f32", out="f32"),
        # the forward of the MLP's first projection in a step of 4096 tokens
        dict(name="prod forward, 7B MLP", op="prod", way="fwd", rows=4096, n=4096, m=11008, fmt="e4m3", out="bf16"),
        # the 13B MLP's input gradient of a short ragged batch, gradients in E5M2
        dict(name="prod input grad, 777 rows", op="prod", way="dx", rows=777, n=5120, m=13824, fmt="e5m2", out="bf16"),
        # the weight gradient of an attention projection, left in 32 bits for the optimizer
        dict(name="prod weight grad, 7B", op="prod", way="dw", rows=4096, n=4096, m=4096, fmt="e4m3", out="f32"),
        # the adapter gradients of the seven projections of a block (rank 64), 32 bits as the backward leaves them
        dict(name="ortho, 7 adapters, f32", op="ortho", batch=7, rows=4096, cols=64, dtype="f32"),
        # a small layer of odd sizes
        dict(name="ortho, odd, f32", op="ortho", batch=1, rows=1000, cols=1531, dtype="f32"),
        # an attention projection's update
        dict(name="ortho, 7B attention", op="ortho", batch=1, rows=4096, cols=4096, dtype="bf16"),
        # an MLP projection's update, tall: the largest
        dict(name="ortho, 7B MLP", op="ortho", batch=1, rows=11008, cols=4096, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _by_16(rng, lo, hi):
    """A layer's width: mostly a multiple of 128, else of 16."""
    v = _log_int(rng, lo, hi)
    return max(lo, v // 128 * 128 if rng.random() < 0.5 else v // 16 * 16)


def draw(rng: random.Random):
    op = rng.choice(["quant", "linear", "prod", "prod", "ortho", "ortho"])
    if op == "quant":
        cols = _log_int(rng, 16, 16384)
        cols = cols if rng.random() < 0.4 else max(16, cols // 16 * 16)
        rows = min(_log_int(rng, 1, 16384), (1 << 26) // cols)
        return dict(op=op, way=rng.choice(["row", "col", "both", "tile"]), rows=rows, cols=cols, dtype=rng.choice(["bf16", "f32"]), fmt=rng.choice(["e4m3", "e4m3", "e5m2"]))
    if op == "linear":
        return dict(op=op, rows=rng.choice([1, 1, _log_int(rng, 1, 64)]), n=_by_16(rng, 128, 14336), m=_by_16(rng, 128, 14336), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    out=rng.choice(["bf16", "bf16", "f32"]))
    if op == "prod":
        n, m = _by_16(rng, 128, 14336), _by_16(rng, 128, 14336)
        return dict(op=op, way=rng.choice(["fwd", "dx", "dw"]), rows=max(1, min(_log_int(rng, 16, 16384), (1 << 39) // (2 * n * m))), n=n, m=m,
                    fmt=rng.choice(["e4m3", "e5m2"]), out=rng.choice(["bf16", "f32"]))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if rng.random() < 0.4:      # adapters: a rank on one side, batches
        short, long, batch = rng.choice([8, 16, 32, 64, 128, _log_int(rng, 4, 256)]), _log_int(rng, 512, 14336), rng.randint(1, 16)
    else:
        short, long, batch = _log_int(rng, 64, 4096), _log_int(rng, 64, 11008), 1
    rows, cols = rng.choice([(short, long), (long, short)])
    return dict(op=op, batch=batch, rows=rows, cols=cols, dtype=dtype)


def _blocks(v):
    return -(-v // BLOCK)


def work(case):
    if case["op"] == "ortho":
        short, long = sorted((case["rows"], case["cols"]))
        size = 2 if case["dtype"] == "bf16" else 4
        # the Gram matrix and its square are symmetric: half of each
        return {"bytes": 2 * case["batch"] * short * long * size, "flops": case["batch"] * STEPS * (3 * short * short * long + short ** 3)}
    if case["op"] == "quant":
        rows, cols, size = case["rows"], case["cols"], 2 if case["dtype"] == "bf16" else 4
        scales = {"row": rows * _blocks(cols), "col": _blocks(rows) * cols, "tile": _blocks(rows) * _blocks(cols)}
        written = rows * cols * (2 if case["way"] == "both" else 1) + (scales["row"] + scales["col"] if case["way"] == "both" else scales[case["way"]])
        return {"bytes": rows * cols * size + written, "flops": 3 * rows * cols}
    rows, n, m = case["rows"], case["n"], case["m"]
    out = 2 if case["out"] == "bf16" else 4
    flops = 2 * rows * n * m
    if case["op"] == "linear":
        return {"bytes": rows * n * (2 if case["dtype"] == "bf16" else 4) + n * m + rows * m * out, "flops": flops}
    sizes = {"x": rows * n, "y": rows * m, "w": n * m}
    result = {"fwd": "y", "dx": "x", "dw": "w"}[case["way"]]
    return {"bytes": sum(sizes.values()) - sizes[result] + sizes[result] * out, "flops": flops}


# ---------------------------------------------------------------------------------------------------------------- the inputs
def _activations(gen, rows, cols, dtype):
    """Normal values with a few large channels, as a block's input has."""
    x = torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.float32)
    loud = torch.randint(0, cols, (max(1, cols // 256),), generator=gen, device="cuda")
    x[:, loud] *= 20.0
    return x.to(dtype)


def _gradients(gen, rows, cols, dtype):
    """Normal values whose size differs from row to row."""
    x = torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.float32)
    return (x * torch.exp(torch.randn((rows, 1), generator=gen, device="cuda") * 1.5 - 7.0)).to(dtype)


def _weights(gen, rows, cols):
    return torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.float32).mul_(0.02)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "ortho":
        # momentum of a gradient: a strong part of low rank with falling weights, and noise
        b, rows, cols = case["batch"], case["rows"], case["cols"]
        k = min(rows, cols, 32)
        fall = 1.0 / torch.arange(1, k + 1, device="cuda", dtype=torch.float32)
        strong = torch.randn((b, rows, k), generator=gen, device="cuda") * fall @ torch.randn((b, k, cols), generator=gen, device="cuda")
        s["x"] = (strong + 0.5 * torch.randn((b, rows, cols), generator=gen, device="cuda")).mul_(1e-3).to(DTYPES[case["dtype"]])
        if b == 1:
            s["x"] = s["x"][0]
        return s
    if case["op"] == "quant":
        make = {"both": _activations, "row": _activations, "col": _gradients}.get(case["way"])
        s["x"] = _weights(gen, case["rows"], case["cols"]).to(DTYPES[case["dtype"]]) if make is None else make(gen, case["rows"], case["cols"], DTYPES[case["dtype"]])
        return s
    rows, n, m = case["rows"], case["n"], case["m"]
    if case["op"] == "linear":
        s["x"] = _activations(gen, rows, n, DTYPES[case["dtype"]])
        s["w"] = _encode(_weights(gen, m, n), "tile", "e4m3")
    elif case["way"] == "fwd":
        s["x"] = _encode(_activations(gen, rows, n, torch.float32), "row", case["fmt"])
        s["w"] = _encode(_weights(gen, m, n), "tile", "e4m3")
    elif case["way"] == "dx":
        s["dy"] = _encode(_gradients(gen, rows, m, torch.float32), "row", case["fmt"])
        s["w"] = _encode(_weights(gen, m, n), "tile", "e4m3")
    else:
        s["dy"] = _encode(_gradients(gen, rows, m, torch.float32), "col", case["fmt"])
        s["x"] = _encode(_activations(gen, rows, n, torch.float32), "col", "e4m3")
    return s


# ---------------------------------------------------------------------------------------------------------------- the plain forms
def _extent(along):
    """Rows and columns of a block."""
    return {"row": (1, BLOCK), "col": (BLOCK, 1), "tile": (BLOCK, BLOCK)}[along]


def _encode(x, along, fmt):
    """8-bit codes of 32-bit x [rows, cols] and the exponent byte of each block: the smallest power of two that brings the block's
    largest value to the type's largest or below."""
    rows, cols = x.shape
    br, bc = _extent(along)
    blocks = torch.nn.functional.pad(x, (0, -cols % bc, 0, -rows % br)).view(-(-rows // br), br, -(-cols // bc), bc)
    mantissa, exponent = torch.frexp(blocks.abs().amax((1, 3)))          # amax = mantissa * 2^exponent, 0.5 <= mantissa < 1
    e = torch.clamp(exponent - (TOP_EXPONENT[fmt] + 1) + (mantissa > 0.875) + 127, min=0) * (mantissa > 0)
    scaled = torch.ldexp(blocks, (127 - e)[:, None, :, None]).view(-(-rows // br) * br, -1)[:rows, :cols]
    return scaled.to(CODES[fmt]).contiguous(), e.to(torch.uint8)


def _decode(q, along):
    codes, scales = q
    br, bc = _extent(along)
    e = (scales.to(torch.int32) - 127).repeat_interleave(br, 0)[:codes.shape[0]].repeat_interleave(bc, 1)[:, :codes.shape[1]]
    return torch.ldexp(codes.float(), e)


def _plain(s, case):
    if case["op"] == "quant":
        x = s["x"].float()
        ways = ["row", "col"] if case["way"] == "both" else [case["way"]]
        return {w: _encode(x, w, case["fmt"]) for w in ways}
    if case["op"] == "linear":
        x = _decode(_encode(s["x"].float(), "row", "e4m3"), "row")
        return (x @ _decode(s["w"], "tile").mT).to(DTYPES[case["out"]])
    if case["op"] == "prod":
        if case["way"] == "fwd":
            r = _decode(s["x"], "row") @ _decode(s["w"], "tile").mT
        elif case["way"] == "dx":
            r = _decode(s["dy"], "row") @ _decode(s["w"], "tile")
        else:
            r = _decode(s["dy"], "col").mT @ _decode(s["x"], "col")
        return r.to(DTYPES[case["out"]])
    x = s["x"].float()
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    x = x / (torch.sqrt(x.double().square().sum((-2, -1), keepdim=True)) + EPS).float()
    a, b, c = QUINTIC
    for _ in range(STEPS):
        g = x @ x.mT
        x = a * x + (b * g + c * (g @ g)) @ x
    return (x.mT if tall else x).to(s["x"].dtype).contiguous()


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if not own:
        return _plain(state, case)
    from paper_2510_24061_b200 import dense
    s = state
    if case["op"] == "quant":
        if case["way"] == "both":
            row, col = dense.block_quantize_both(s["x"], fmt=case["fmt"])
            return {"row": (row.codes, row.scales), "col": (col.codes, col.scales)}
        q = dense.block_quantize(s["x"], along=case["way"], fmt=case["fmt"])
        return {case["way"]: (q.codes, q.scales)}
    if case["op"] == "linear":
        return dense.block_forward(s["x"], dense.Blocks(*s["w"], "tile"), dtype=DTYPES[case["out"]])
    if case["op"] == "prod":
        if case["way"] == "fwd":
            return dense.block_forward(dense.Blocks(*s["x"], "row"), dense.Blocks(*s["w"], "tile"), dtype=DTYPES[case["out"]])
        if case["way"] == "dx":
            return dense.block_input_grad(dense.Blocks(*s["dy"], "row"), dense.Blocks(*s["w"], "tile"), dtype=DTYPES[case["out"]])
        return dense.block_weight_grad(dense.Blocks(*s["dy"], "col"), dense.Blocks(*s["x"], "col"), dtype=DTYPES[case["out"]])
    return dense.orthogonalize(s["x"], steps=STEPS, eps=EPS)


# ---------------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_round(v, fmt):
    """The nearest value of the 8-bit type (ties to the even one) of 64-bit v within its range."""
    digits, low = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
    _, e = torch.frexp(v)
    spacing = torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=low) - digits)
    return torch.round(v / spacing) * spacing


def _exact_blocks(x, along, fmt):
    """(values of the codes, exponents of the blocks spread over the values) of 64-bit x."""
    rows, cols = x.shape
    br, bc = _extent(along)
    at_r, at_c = torch.arange(rows, device=x.device) // br, torch.arange(cols, device=x.device) // bc
    amax = torch.zeros((int(at_r[-1]) + 1, cols), dtype=torch.float64, device=x.device).index_reduce_(0, at_r, x.abs(), "amax")
    amax = torch.zeros((amax.shape[0], int(at_c[-1]) + 1), dtype=torch.float64, device=x.device).index_reduce_(1, at_c, amax, "amax")
    top = 1.75 * 2.0 ** TOP_EXPONENT[fmt]
    p = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -200) / top))
    p = torch.where(amax > top * torch.exp2(p), p + 1, p)              # log2 may be off by a rounding at a power of two
    p = torch.where(amax <= top * torch.exp2(p - 1), p - 1, p).clamp(min=-127)
    p = p[at_r][:, at_c]
    return _exact_round(x / torch.exp2(p), fmt), p


def _exact_value(q, along):
    codes, scales = q
    br, bc = _extent(along)
    at_r, at_c = torch.arange(codes.shape[0], device=codes.device) // br, torch.arange(codes.shape[1], device=codes.device) // bc
    return codes.double() * torch.exp2(scales.double() - 127.0)[at_r][:, at_c]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quant":
        ways = ["row", "col"] if case["way"] == "both" else [case["way"]]
        return {w: (_exact_blocks(s["x"].double(), w, case["fmt"])[0], None) for w in ways}
    if case["op"] == "linear":
        codes, p = _exact_blocks(s["x"].double(), "row", "e4m3")
        return torch.einsum("tn,mn->tm", codes * torch.exp2(p), _exact_value(s["w"], "tile"))
    if case["op"] == "prod":
        if case["way"] == "fwd":
            return torch.einsum("tn,mn->tm", _exact_value(s["x"], "row"), _exact_value(s["w"], "tile"))
        if case["way"] == "dx":
            return torch.einsum("tm,mn->tn", _exact_value(s["dy"], "row"), _exact_value(s["w"], "tile"))
        return torch.einsum("tm,tn->mn", _exact_value(s["dy"], "col"), _exact_value(s["x"], "col"))
    x = s["x"].double()
    tall = x.shape[-2] > x.shape[-1]
    a, b, c = QUINTIC
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    eye = torch.eye(min(x.shape[-2:]), dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        # p(G) = a + b G + c G^2 by Horner's rule, applied from the short side
        g = torch.matmul(x.mT, x) if tall else torch.matmul(x, x.mT)
        p = torch.matmul(g, c * g + b * eye) + a * eye
        x = torch.matmul(x, p) if tall else torch.matmul(p, x)
    return x
