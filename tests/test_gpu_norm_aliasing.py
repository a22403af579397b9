"""Block norms in place, as the header allows it, and calls that want a part of the results only: the same bits as with buffers of their own."""
import pytest
import torch

from tests import train_oracle as orc
from tests.test_gpu_block_norm import close, inputs, on_gpu, reference

pytestmark = pytest.mark.gpu

# every kernel: whole spans, other multiples of 16, odd widths, rows that no shared memory holds; runs that begin and end inside 16-byte pieces
SIZES = [(700, 1024, 100), (300, 5120, 300), (450, 96, 7), (310, 1000, 155), (613, 1011, 123), (450, 5001, 225), (9, 16384, 4), (7, 14501, 3), (1, 4096, 1), (400, 33, 400)]


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,rpg", SIZES)
def test_forward_in_place(tr, rows, cols, rpg, dtype):
    t, kw = inputs(rows, cols, rpg, True, True, True, True, dtype, torch.float32, 21)
    kw = on_gpu(kw)
    want = tr.block_norm_forward(t["h"].cuda(), t["y"].cuda(), save=True, **kw)
    for place in ("h", "y"):
        g = {k: t[k].cuda() for k in ("h", "y")}
        out = tr.block_norm_forward(g["h"], g["y"], save=True, h_out=g[place], **kw)
        assert out.h_out.data_ptr() == g[place].data_ptr()
        for a, b in zip(out, want):
            for p, q in zip(a if isinstance(a, tuple) else (a,), b if isinstance(b, tuple) else (b,)):
                assert torch.equal(p, q), place


@pytest.mark.parametrize("saved", ["codes", "plain"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,rpg", SIZES)
def test_backward_in_place(tr, rows, cols, rpg, dtype, saved):
    t, kw = inputs(rows, cols, rpg, True, True, True, True, dtype, torch.float32, 22)
    g, kw = {k: v.cuda() for k, v in t.items()}, on_gpu(kw)
    out = tr.block_norm_forward(g["h"], g["y"], save=saved == "codes", **kw)
    kept = (out.saved_h, out.saved_y) if saved == "codes" else (g["h"], g["y"])
    want = tr.block_norm_backward(g["dx"], g["dh_out"], *kept, out.inv_post, out.inv_pre, **kw)
    for dh, dy in (("dx", "dh_out"), ("dh_out", "dx"), ("dx", None), ("dh_out", None), (None, "dx")):
        b = {k: g[k].clone() for k in ("dx", "dh_out")}
        got = tr.block_norm_backward(b["dx"], b["dh_out"], *kept, out.inv_post, out.inv_pre, dh=b.get(dh), dy=b.get(dy), **kw)
        for name, p, q in zip(want._fields, got, want):
            assert torch.equal(p, q), (dh, dy, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,rpg", SIZES)
def test_forward_without_the_residual_stream(tr, rows, cols, rpg, dtype):
    """Only x is wanted: what it is does not depend on it (another kernel may run: the same roundings in another order of the sums)."""
    t, kw = inputs(rows, cols, rpg, True, True, True, True, dtype, torch.float32, 23)
    ref = reference(rows, cols, kw)
    H, x = ref.forward(orc.d(t["h"]), orc.d(t["y"]))
    out = tr.block_norm_forward(t["h"].cuda(), t["y"].cuda(), need_h_out=False, save=True, **on_gpu(kw))
    assert out.h_out is None and out.saved_h is not None
    spread = 1 + (ref.H_size ** 2).mean(1, keepdim=True) / ((H ** 2).mean(1, keepdim=True) + kw["eps"])
    close(out.x, x, ref.H_size * ref.iq * ref.w2.abs() * spread, dtype, 64)


@pytest.mark.parametrize("saved", ["codes", "plain"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,rpg", SIZES)
def test_backward_of_some_results(tr, rows, cols, rpg, dtype, saved):
    """Every choice of gradients, each against 64 bits; what is not asked for is not there."""
    t, kw = inputs(rows, cols, rpg, True, True, True, True, dtype, torch.float32, 24)
    g, kg = {k: v.cuda() for k, v in t.items()}, on_gpu(kw)
    out = tr.block_norm_forward(g["h"], g["y"], save=saved == "codes", **kg)
    kept = (out.saved_h, out.saved_y) if saved == "codes" else (g["h"], g["y"])
    hd, yd = (torch.from_numpy(orc.decode(v.codes.cpu().numpy(), v.scales.cpu().numpy())) if saved == "codes" else orc.d(v) for v in kept)
    ref = reference(rows, cols, kw).backward(orc.d(t["dx"]), orc.d(t["dh_out"]), hd, yd, orc.d(out.inv_post), orc.d(out.inv_pre))
    for need_dy, gains in ((False, True), (False, False), (True, ("gate",)), (True, ("pre_gain",)), (False, ("post_gain",)), (True, ("post_gain", "pre_gain"))):
        got = tr.block_norm_backward(g["dx"], g["dh_out"], *kept, out.inv_post, out.inv_pre, need_dy=need_dy, need_gains=gains, **kg)
        names = ("post_gain", "pre_gain", "gate") if gains is True else gains or ()
        assert (got.dy is not None) == need_dy and [n for n in ("post_gain", "pre_gain", "gate") if getattr(got, "d" + n) is not None] == sorted(names, key=("post_gain", "pre_gain", "gate").index)
        for name in ("dh", "dy"):
            if getattr(got, name) is not None:
                close(getattr(got, name), *ref[name], dtype, 64)
        for name in names:
            close(getattr(got, "d" + name), *ref["d" + name], torch.float32, 64 + min(rows, 700))
