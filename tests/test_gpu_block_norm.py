"""The norms after and before a block with its gate and the residual scale, forward and backward, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import train_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


# rows, cols, rows per gate row (0: no gate), post, pre, residual, gains: one token to several CTAs' worth; widths of one value, of
# single columns (7, 1011), of whole vectors without whole checkpoint blocks (40, 1000), and the widest; ragged gate groups
CASES = [
    (1, 4096, 1, True, True, True, True), (1, 1, 1, True, True, True, True), (5, 7, 2, True, True, True, True),
    (300, 64, 0, True, True, True, True), (37, 40, 5, True, True, True, False), (150, 512, 150, True, True, True, True),
    (613, 1011, 123, True, True, True, True), (33, 1000, 33, False, True, True, True), (64, 2048, 64, True, False, True, True),
    (129, 4096, 129, True, True, True, True), (40, 4112, 7, True, True, False, True), (300, 5120, 100, True, True, True, True),
    (9, 8192, 9, True, True, True, True), (6, 11008, 2, True, True, True, True), (5, 16384, 5, True, True, True, True),
    (7, 16383, 3, True, True, True, True), (257, 256, 1, True, True, True, True), (20, 96, 0, False, False, True, False),
    (700, 1536, 64, True, True, True, True), (16, 128, 16, False, True, False, False),
    (1, 4095, 1, True, True, True, True), (17, 2049, 6, True, True, True, True), (5, 5111, 2, True, False, True, True), (3, 8191, 3, False, True, True, False),
    (2, 9, 2, True, True, False, True), (400, 33, 0, True, True, True, True), (2, 6160, 1, True, True, True, True), (3, 12300, 3, True, True, True, True),
    (310, 9001, 155, True, True, True, True), (450, 5001, 225, True, True, True, True), (160, 8208, 0, True, True, True, True),
]
IDS = [f"{c[0]}x{c[1]}" for c in CASES]


def inputs(rows, cols, rpg, post, pre, residual, gains, dtype, gain_dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    n = lambda shape, s: torch.randn(shape, generator=gen) * s  # noqa: E731
    t = dict(y=n((rows, cols), 0.7).to(dtype), h=n((rows, cols), 2.0).to(dtype) if residual else None,
             dx=n((rows, cols), 1e-2).to(dtype) if pre else None, dh_out=n((rows, cols), 1e-2).to(dtype))
    kw = dict(post=post, pre=pre, res_scale=0.75, gain_offset=0.0 if gain_dtype == torch.float32 else 1.0, eps=1e-5)
    if gains and post:
        kw["post_gain"] = (n((cols,), 0.1) + (1.0 - kw["gain_offset"])).to(gain_dtype)
    if gains and pre:
        kw["pre_gain"] = (n((cols,), 0.1) + (1.0 - kw["gain_offset"])).to(gain_dtype)
    if rpg:
        kw["gate"], kw["rows_per_gate"] = (n((-(-rows // rpg), cols), 0.3) + 0.5).to(gain_dtype), rpg
    return t, kw


def on_gpu(kw):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}


def reference(rows, cols, kw):
    return orc.Norm(rows, cols, **{k: orc.d(v) if isinstance(v, torch.Tensor) else v for k, v in kw.items()})


def close(got, want, size, dtype, fp32_steps):
    """|got - want| <= fp32_steps * 2^-24 * (sum of the magnitudes that went in) + the rounding of the stored type."""
    tol = fp32_steps * 2.0 ** -24 * size + orc.type_rounding(dtype) * (want.abs() + fp32_steps * 2.0 ** -24 * size) + 1e-38
    err = (got.cpu().double() - want).abs()
    assert torch.isfinite(got).all() and (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dtype,gain_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(tr, case, dtype, gain_dtype):
    t, kw = inputs(*case, dtype, gain_dtype, 7)
    rows, cols = t["y"].shape
    ref = reference(rows, cols, kw)
    H, x = ref.forward(orc.d(t["h"]), orc.d(t["y"]))
    amax = torch.zeros(1, device="cuda")
    out = tr.block_norm_forward(None if t["h"] is None else t["h"].cuda(), t["y"].cuda(), save=True, amax_x=amax, **on_gpu(kw))
    # the squares' sum is a tree over at most 16 values a thread, 32 lanes and 32 warps (26 roundings), the root 2 more; a value then
    # takes at most 6 operations: 32 units in the last place of what went in bound h_out, twice that x
    close(out.h_out, H, ref.H_size, dtype, 32)
    if kw["post"]:
        close(out.inv_post, ref.ip[:, 0], ref.ip[:, 0], torch.float32, 32)
    else:
        assert out.inv_post is None
    if kw["pre"]:
        close(out.inv_pre, ref.iq[:, 0], ref.iq[:, 0] * 2 * (ref.H_size ** 2).mean(1) / ((H ** 2).mean(1) + kw["eps"]), torch.float32, 64)
        spread = 1 + (ref.H_size ** 2).mean(1, keepdim=True) / ((H ** 2).mean(1, keepdim=True) + kw["eps"])
        close(out.x, x, ref.H_size * ref.iq * ref.w2.abs() * spread, dtype, 64)
        assert amax.item() == out.x.float().abs().max().item()
    else:
        assert out.x is None and out.inv_pre is None and amax.item() == 0
    for ck, v in ((out.saved_h, t["h"]), (out.saved_y, t["y"])):
        if v is None:
            assert ck is None
            continue
        e, vals = orc.encode(v.double().numpy())
        assert np.array_equal(ck.scales.cpu().numpy(), e) and np.array_equal(orc.e4m3_values()[ck.codes.cpu().numpy()], vals)
    again = tr.block_norm_forward(None if t["h"] is None else t["h"].cuda(), t["y"].cuda(), **on_gpu(kw))
    assert torch.equal(again.h_out, out.h_out) and (out.x is None or torch.equal(again.x, out.x)) and again.saved_y is None


@pytest.mark.parametrize("saved", ["codes", "plain"])
@pytest.mark.parametrize("dtype,gain_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(tr, case, dtype, gain_dtype, saved):
    t, kw = inputs(*case, dtype, gain_dtype, 11)
    rows, cols = t["y"].shape
    g = {k: None if v is None else v.cuda() for k, v in t.items()}
    out = tr.block_norm_forward(g["h"], g["y"], save=saved == "codes", **on_gpu(kw))
    if saved == "codes":
        h, y = out.saved_h, out.saved_y
        hd, yd = (None if k is None else torch.from_numpy(orc.decode(k.codes.cpu().numpy(), k.scales.cpu().numpy())) for k in (h, y))
    else:
        h, y, hd, yd = g["h"], g["y"], orc.d(t["h"]), orc.d(t["y"])
    amax = torch.zeros(1, device="cuda")
    got = tr.block_norm_backward(g["dx"], g["dh_out"], h, y, out.inv_post, out.inv_pre, amax_dy=amax, **on_gpu(kw))
    ref = reference(rows, cols, kw).backward(orc.d(t["dx"]), orc.d(t["dh_out"]), hd, yd, orc.d(out.inv_post), orc.d(out.inv_pre))
    # row sums: 26 roundings as in the forward and a dozen operations per value: 64 units in the last place of the magnitudes;
    # column sums: at most rows_per_unit + 148 / 8 + 8 additions more, and 700 rows at the most here
    for name in ("dh", "dy"):
        have = getattr(got, name)
        if name == "dh" and t["h"] is None:
            assert have is None
            continue
        close(have, *ref[name], dtype, 64)
    for name, there in (("dpost_gain", "post_gain" in kw), ("dpre_gain", "pre_gain" in kw), ("dgate", "gate" in kw)):
        have = getattr(got, name)
        assert (have is not None) == there
        if there:
            close(have, *ref[name], torch.float32, 64 + min(rows, 700))
    assert amax.item() == got.dy.float().abs().max().item()
    # the same bits again; frozen gains change nothing else; in place
    more = tr.block_norm_backward(g["dx"], g["dh_out"], h, y, out.inv_post, out.inv_pre, **on_gpu(kw))
    frozen = tr.block_norm_backward(g["dx"], g["dh_out"], h, y, out.inv_post, out.inv_pre, need_gains=False, **on_gpu(kw))
    for a, b, c in zip(got, more, frozen):
        assert a is None or torch.equal(a, b)
        assert a is None or c is None or torch.equal(a, c)
    assert frozen.dpost_gain is None and frozen.dgate is None
    into = g["dh_out"].clone()
    first = tr.block_norm_backward(g["dx"], into, h, y, out.inv_post, out.inv_pre, need_gains=False, dy=into, **on_gpu(kw))
    assert torch.equal(first.dy, got.dy) and first.dy.data_ptr() == into.data_ptr()


def test_gradient_against_differences(tr):
    """Directional derivatives of the 64-bit forward by central differences: dh, dy, gains and gate together."""
    rows, cols, rpg = 12, 48, 5
    t, kw = inputs(rows, cols, rpg, True, True, True, True, torch.float32, torch.float32, 3)
    out = tr.block_norm_forward(t["h"].cuda(), t["y"].cuda(), **on_gpu(kw))
    got = tr.block_norm_backward(t["dx"].cuda(), t["dh_out"].cuda(), t["h"].cuda(), t["y"].cuda(), out.inv_post, out.inv_pre, **on_gpu(kw))
    gen = torch.Generator().manual_seed(1)
    v = {k: torch.randn(s.shape, generator=gen, dtype=torch.float64) for k, s in (("h", t["h"]), ("y", t["y"]), ("post_gain", kw["post_gain"]), ("pre_gain", kw["pre_gain"]), ("gate", kw["gate"]))}

    def f(s):
        at = {k: (orc.d(t[k]) if k in ("h", "y") else orc.d(kw[k])) + s * v[k] for k in v}
        ref = orc.Norm(rows, cols, **{k: at.get(k, w) for k, w in kw.items()})
        H, x = ref.forward(at["h"], at["y"])
        return float((H * orc.d(t["dh_out"])).sum() + (x * orc.d(t["dx"])).sum())

    step = 1e-5
    want = (f(step) - f(-step)) / (2 * step)
    terms = [(got.dh, "h"), (got.dy, "y"), (got.dpost_gain, "post_gain"), (got.dpre_gain, "pre_gain"), (got.dgate, "gate")]
    have = sum(float((orc.d(g) * v[k]).sum()) for g, k in terms)
    size = sum(float((orc.d(g) * v[k]).abs().sum()) for g, k in terms)
    assert abs(have - want) <= 1e-5 * size      # fp32 gradients (1e-6) and the differences' own step^2 = 1e-10 and 1e-16 / step


def test_a_zero_row_and_large_values(tr):
    """A row of zeros divides by sqrt(eps) only; rows of 1e18 keep their squares in range."""
    for cols in (512, 37):
        y, h = torch.zeros((3, cols)), torch.zeros((3, cols))
        y[1], h[1] = 1e18, -1e18
        y[2] = torch.arange(cols).float()
        out = tr.block_norm_forward(h.cuda(), y.cuda(), post=True, pre=True, eps=1e-6, save=True)
        ref = orc.Norm(3, cols)
        H, x = ref.forward(h.double(), y.double())
        for got, want in ((out.h_out, H), (out.x, x)):
            assert torch.isfinite(got).all()
            assert torch.allclose(got.cpu().double(), want, rtol=1e-5, atol=0)
        g = tr.block_norm_backward(torch.ones((3, cols), device="cuda"), None, out.saved_h, out.saved_y, out.inv_post, out.inv_pre)
        assert torch.isfinite(g.dh).all() and torch.isfinite(g.dy).all()


def test_nan_stays_in_its_row(tr):
    for cols in (256, 45):
        h, y = torch.randn((4, cols)), torch.randn((4, cols))
        y[2, 3] = float("nan")
        out = tr.block_norm_forward(h.cuda(), y.cuda(), save=True)
        assert torch.isnan(out.h_out[2]).all() and torch.isnan(out.x[2]).all()
        keep = torch.tensor([0, 1, 3])
        assert torch.isfinite(out.h_out.cpu()[keep]).all() and torch.isfinite(out.x.cpu()[keep]).all()


def test_another_stream_and_a_captured_graph(tr):
    t, kw = inputs(200, 1024, 50, True, True, True, True, torch.bfloat16, torch.bfloat16, 5)
    g, kw = {k: v.cuda() for k, v in t.items()}, on_gpu(kw)
    out = tr.block_norm_forward(g["h"], g["y"], save=True, **kw)
    want = tr.block_norm_backward(g["dx"], g["dh_out"], out.saved_h, out.saved_y, out.inv_post, out.inv_pre, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o = tr.block_norm_forward(g["h"], g["y"], save=True, **kw)
        b = tr.block_norm_backward(g["dx"], g["dh_out"], o.saved_h, o.saved_y, o.inv_post, o.inv_pre, **kw)
    side.synchronize()
    assert torch.equal(o.x, out.x) and all(torch.equal(p, q) for p, q in zip(b, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = tr.block_norm_forward(g["h"], g["y"], save=True, **kw)
        b = tr.block_norm_backward(g["dx"], g["dh_out"], o.saved_h, o.saved_y, o.inv_post, o.inv_pre, **kw)
    for _ in range(3):
        for v in b:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o.x, out.x) and all(torch.equal(p, q) for p, q in zip(b, want))
