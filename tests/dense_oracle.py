"""The operators of include/falqon_dense.h in 64 bits, from their definitions."""
import torch

BLOCK = 128
TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
QUINTIC = (3.4445, -4.7750, 2.0315)


def extent(along):
    return {"row": (1, BLOCK), "col": (BLOCK, 1), "tile": (BLOCK, BLOCK)}[along]


def spread(scales, along, rows, cols):
    """A value per block, given to each value of the block."""
    br, bc = extent(along)
    dev = scales.device
    return scales[torch.arange(rows, device=dev) // br][:, torch.arange(cols, device=dev) // bc]


def scale_bytes(x, along, fmt):
    """The smallest e >= 0 with amax * 2^(127 - e) <= top; 255 where a block holds an infinity or a NaN."""
    rows, cols = x.shape
    br, bc = extent(along)
    full = torch.zeros((-(-rows // br) * br, -(-cols // bc) * bc), dtype=torch.float64, device=x.device)
    full[:rows, :cols] = x.double()
    blocks = full.view(full.shape[0] // br, br, full.shape[1] // bc, bc).abs()
    bad = ~torch.isfinite(blocks).all(3).all(1)
    amax = torch.where(bad, 0.0, blocks.nan_to_num(0.0, 0.0).amax((1, 3)))
    e = torch.zeros_like(amax)
    for k in range(255):        # from the definition, one exponent after the other
        e = torch.where(amax * 2.0 ** (127 - k) > TOP[fmt], k + 1.0, e)
    return torch.where(bad, 255.0, e).to(torch.uint8)


def round_to(v, fmt):
    """The nearest value of the 8-bit type, ties to even, of |v| <= top."""
    digits, low = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=low) - digits)
    return torch.round(v / step) * step


def quantize(x, along, fmt):
    """(values of the codes in 64 bits, scale bytes); NaN in blocks marked 255."""
    e = scale_bytes(x, along, fmt)
    each = spread(e, along, *x.shape).double()
    v = round_to(torch.where(each == 255, 0.0, x.double()) * torch.exp2(127.0 - each), fmt)
    return torch.where(each == 255, float("nan"), v), e


def value(q):
    """What Blocks stand for."""
    codes, scales, along = q
    each = spread(scales, along, *codes.shape).double()
    return torch.where(each == 255, float("nan"), codes.double() * torch.exp2(each - 127.0))


def orthogonalize(g, coefficients, eps, scale=1.0):
    x = g.double()
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for a, b, c in coefficients:
        m = x @ x.mT
        x = a * x + (b * m + c * (m @ m)) @ x
    return scale * (x.mT if tall else x)
