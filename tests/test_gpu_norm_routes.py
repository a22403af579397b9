"""Which kernels the block norms launch: the staged ones wherever a row fits in shared memory, on every CTA that can be resident."""
import pytest
import torch

from tests.launches import launched

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


def one(n, v=1.0):
    return torch.full((n,), v, device="cuda")


def backward_call(tr, rows, cols, rpg, dtype, coded, gains=True):
    h, y, dx, dh_out = (torch.randn((rows, cols), device="cuda").to(dtype) for _ in range(4))
    gates = -(-rows // rpg)
    kw = dict(post_gain=one(cols), pre_gain=one(cols), gate=torch.rand((gates, cols), device="cuda"), rows_per_gate=rpg, res_scale=0.5)
    out = tr.block_norm_forward(h, y, save=coded, **kw)
    saved = (out.saved_h, out.saved_y) if coded else (h, y)
    return lambda: tr.block_norm_backward(dx, dh_out, *saved, out.inv_post, out.inv_pre, need_gains=gains, **kw)


@pytest.mark.parametrize("gains", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("rows,cols,rpg", [(724, 256, 724), (1, 1024, 1), (300, 64, 300), (37, 40, 5), (257, 256, 1), (16, 128, 16), (1000, 1024, 1), (200, 512, 200),
                                           (150, 97, 150), (5, 1, 5), (1, 16, 1), (400, 33, 100)])
def test_short_runs_of_narrow_rows_are_staged(tr, rows, cols, rpg, dtype, coded, gains):
    """Few rows per CTA, and rows of one to a few spans: the warps that could share a run's columns are more than its rows."""
    names = [n for n, _, _ in launched(backward_call(tr, rows, cols, rpg, dtype, coded, gains)) if "norm_backward" in n]
    assert len(names) == 1 and "norm_backward_run_kernel" in names[0]


# saved values, width, whether rows of it are staged: both sides of each limit
LIMITS = [("bf16", True, 16350, True), ("bf16", True, 16351, False), ("bf16", True, 16384, True), ("bf16", False, 14431, True), ("bf16", False, 14433, False),
          ("bf16", False, 16384, True), ("f32", True, 12742, True), ("f32", True, 12743, False), ("f32", True, 16384, True), ("f32", False, 14336, True),
          ("f32", False, 14432, True), ("f32", False, 14448, False), ("f32", False, 9623, True), ("f32", False, 9625, False)]


@pytest.mark.parametrize("dtype,coded,cols,staged", LIMITS)
def test_the_widest_rows(tr, dtype, coded, cols, staged):
    """On each side of the widths up to which a row is staged: the kernel, and the gradients against 64 bits."""
    from tests import test_gpu_block_norm as norm
    from tests import train_oracle as orc
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    names = [n for n, _, _ in launched(backward_call(tr, 3, cols, 2, dt, coded)) if "norm_backward" in n]
    assert len(names) == 1 and ("norm_backward_run_kernel" in names[0]) == staged
    t, kw = norm.inputs(3, cols, 2, True, True, True, True, dt, torch.float32, cols)
    g, kg = {k: v.cuda() for k, v in t.items()}, norm.on_gpu(kw)
    out = tr.block_norm_forward(g["h"], g["y"], save=coded, **kg)
    saved = (out.saved_h, out.saved_y) if coded else (g["h"], g["y"])
    got = tr.block_norm_backward(g["dx"], g["dh_out"], *saved, out.inv_post, out.inv_pre, **kg)
    hd, yd = (torch.from_numpy(orc.decode(v.codes.cpu().numpy(), v.scales.cpu().numpy())) if coded else orc.d(v) for v in saved)
    ref = norm.reference(3, cols, kw).backward(orc.d(t["dx"]), orc.d(t["dh_out"]), hd, yd, orc.d(out.inv_post), orc.d(out.inv_pre))
    for name in ("dh", "dy"):
        norm.close(getattr(got, name), *ref[name], dt, 64)
    for name in ("dpost_gain", "dpre_gain", "dgate"):
        norm.close(getattr(got, name), *ref[name], torch.float32, 64 + 3)


FORMS = {"both": {}, "post only": dict(pre=False), "pre only": dict(post=False), "no residual": dict(h=False), "frozen": dict(gate=False)}


def forward_call(tr, rows, cols, dtype, form, save):
    kw = dict(FORMS[form])
    h, y = (torch.randn((rows, cols), device="cuda").to(dtype) for _ in range(2))
    if not kw.pop("h", True):
        h = None
    gate = torch.rand((1, cols), device="cuda") if kw.pop("gate", True) else None
    if kw.get("post", True):
        kw["post_gain"] = one(cols)
    if kw.get("pre", True):
        kw["pre_gain"] = one(cols)
    return lambda: tr.block_norm_forward(h, y, gate=gate, save=save, **kw)


@pytest.mark.parametrize("save", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("cols", [1024, 4096, 4112, 5120, 8192, 9216, 4095])
def test_every_forward_fills_the_gpu(tr, cols, form, dtype, save):
    """As many CTAs as are resident: 148, one to an SM, or 296 of the kernel whose threads take two spans (it is compiled for two to an SM)."""
    (name, ctas, _), = [v for v in launched(forward_call(tr, 2000, cols, dtype, form, save)) if "norm_forward" in v[0]]
    rows = 2000
    two = "norm_forward_rows_kernel" in name and cols <= 8192
    per = -(-rows // (296 if two else 148))
    assert ctas == -(-rows // per)
    usual = form in ("both", "frozen") and cols % 1024 == 0 and cols <= 8192
    if dtype == torch.bfloat16 and cols % 16 == 0:
        assert ("norm_forward_full_kernel" in name) == usual


@pytest.mark.parametrize("dtype,cols,staged", [("bf16", 16383, True), ("f32", 14335, True), ("f32", 14337, False), ("f32", 16384, True)])
def test_the_widest_rows_forward(tr, dtype, cols, staged):
    """Only fp32 rows of odd widths ever leave the staged kernels, on either side of their limit; results against 64 bits."""
    from tests import test_gpu_block_norm as norm
    from tests import train_oracle as orc
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    t, kw = norm.inputs(3, cols, 2, True, True, True, True, dt, torch.float32, cols)
    h, y, kg = t["h"].cuda(), t["y"].cuda(), norm.on_gpu(kw)
    (name, _, _), = launched(lambda: tr.block_norm_forward(h, y, save=True, **kg))
    assert ("norm_forward_f32_kernel" not in name) == staged
    out = tr.block_norm_forward(h, y, save=True, **kg)
    ref = norm.reference(3, cols, kw)
    H, x = ref.forward(orc.d(t["h"]), orc.d(t["y"]))
    norm.close(out.h_out, H, ref.H_size, dt, 32)
    spread = 1 + (ref.H_size ** 2).mean(1, keepdim=True) / ((H ** 2).mean(1, keepdim=True) + kw["eps"])
    norm.close(out.x, x, ref.H_size * ref.iq * ref.w2.abs() * spread, dt, 64)
    e, vals = orc.encode(t["y"].double().numpy())
    assert (out.saved_y.scales.cpu().numpy() == e).all() and (orc.e4m3_values()[out.saved_y.codes.cpu().numpy()] == vals).all()
