"""Host-side checks of include/falqon_train.h that need no GPU: exported symbols, plain C, sizes, refusals before any launch."""
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
def tr():
    from paper_2510_24061_b200 import build
    build.build()
    from paper_2510_24061_b200 import training
    return training


@pytest.fixture(scope="module")
def fq(tr):
    from paper_2510_24061_b200 import binding
    return binding


def test_every_declared_symbol_is_exported_and_bound(tr):
    header = open(os.path.join(ROOT, "include", "falqon_train.h")).read()
    declared = set(re.findall(r"^(?:int|size_t) (falqon_[a-z_]+)\s*\(", header, flags=re.M))
    assert declared == set(tr.TRAIN_EXPORTS)
    for name in declared:
        assert hasattr(tr.lib, name), name


def test_the_header_is_plain_c(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text('#include "falqon_train.h"\nint main(void) { falqon_block_norm n; falqon_preference p; (void)n; (void)p; return 0; }\n')
    for cmd in (["gcc", "-std=c99", "-pedantic"], ["g++", "-std=c++11", "-x", "c++"]):
        subprocess.run([*cmd, "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)], check=True)


def test_struct_layouts_match_the_header(tr, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    fields = {"falqon_block_norm": tr.falqon_block_norm, "falqon_preference": tr.falqon_preference}
    lines = [f'printf("%zu\\n", sizeof({s}));' + "".join(f'printf("%zu\\n", offsetof({s}, {f}));' for f, *_ in t._fields_) for s, t in fields.items()]
    src.write_text('#include <stdio.h>\n#include "falqon_train.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [v for t in fields.values() for v in [C.sizeof(t)] + [getattr(t, f).offset for f, *_ in t._fields_]]
    assert got == want


def test_checkpoint_refusals(fq, tr):
    inv, lib = fq.ERR_INVALID_ARG, tr.lib
    assert lib.falqon_checkpoint_save(None, 0, 4, 8, FAKE, FAKE, None) == inv
    assert lib.falqon_checkpoint_save(FAKE, 2, 4, 8, FAKE, FAKE, None) == inv
    assert lib.falqon_checkpoint_save(FAKE, 0, 0, 8, FAKE, FAKE, None) == inv
    assert lib.falqon_checkpoint_save(FAKE, 0, 4, 0, FAKE, FAKE, None) == inv
    assert lib.falqon_checkpoint_save(FAKE, 0, 1 << 31, 1 << 31, FAKE, FAKE, None) == inv     # more than 2^42 values
    assert lib.falqon_checkpoint_save(FAKE + 2, 0, 4, 8, FAKE, FAKE, None) == inv
    assert lib.falqon_checkpoint_save(FAKE, 0, 4, 8, FAKE + 8, FAKE, None) == inv
    assert lib.falqon_checkpoint_load(FAKE, None, 4, 8, FAKE, 0, None) == inv
    assert lib.falqon_checkpoint_load(FAKE, FAKE, 4, -1, FAKE, 0, None) == inv
    assert lib.falqon_gate_forward(FAKE, None, 0, 4, 8, FAKE, None, None, None, None, None, None) == inv
    assert lib.falqon_gate_forward(FAKE, FAKE, 0, 4, 8, FAKE, FAKE, FAKE, FAKE, None, None, None) == inv    # some of the four
    assert lib.falqon_gate_forward(FAKE, 2 * FAKE, 0, 4, 8, FAKE, None, None, None, None, None, None) == inv      # z is g
    assert lib.falqon_gate_backward(FAKE, FAKE, FAKE, FAKE, FAKE, 0, 4, 8, FAKE, FAKE, None, None, None) == inv   # dg is du
    assert lib.falqon_gate_backward(FAKE, FAKE, FAKE, FAKE, FAKE + 4, 0, 4, 8, FAKE, 2 * FAKE, None, None, None) == inv


def plan(tr, **kw):
    a = dict(rows=8, cols=64, rows_per_gate=8, dtype=0, gain_dtype=1, flags=3, res_scale=1.0, gain_offset=0.0, eps=1e-6, post_gain=FAKE,
             pre_gain=FAKE, gate=FAKE)
    a.update(kw)
    return C.byref(tr.falqon_block_norm(*a.values()))


def test_block_norm_refusals(fq, tr):
    inv, lib = fq.ERR_INVALID_ARG, tr.lib

    def fwd(p, h=FAKE, y=FAKE, h_out=FAKE, x=FAKE, ip=FAKE, iq=FAKE, codes=(None,) * 4):
        return lib.falqon_block_norm_forward(p, h, y, h_out, x, ip, iq, *codes, None, None)

    bad = [dict(rows=0), dict(cols=0), dict(cols=tr.NORM_MAX_COLS + 1), dict(rows_per_gate=0), dict(dtype=2), dict(gain_dtype=-1), dict(flags=4),
           dict(eps=-1.0), dict(eps=float("nan")), dict(res_scale=float("nan")), dict(post_gain=FAKE + 4), dict(gate=FAKE + 8), dict(rows=1 << 31)]
    for kw in bad:
        assert fwd(plan(tr, **kw)) == inv, kw
        assert lib.falqon_block_norm_scratch_bytes(plan(tr, **kw)) == 0
    assert fwd(None) == inv and fwd(plan(tr), y=None) == inv and fwd(plan(tr), x=None) == inv and fwd(plan(tr), iq=None) == inv
    assert fwd(plan(tr), ip=None) == inv and fwd(plan(tr, flags=1), h_out=None) == inv and fwd(plan(tr), y=FAKE + 2) == inv
    assert fwd(plan(tr), codes=(FAKE, None, None, None)) == inv and fwd(plan(tr), h=None, codes=(FAKE, FAKE, None, None)) == inv

    def bwd(p, dx=FAKE, dh_out=FAKE, h=FAKE, hc=(None, None), y=FAKE, yc=(None, None), ip=FAKE, iq=FAKE, dh=FAKE, dy=2 * FAKE, dpost=FAKE,
            dpre=FAKE, dgate=FAKE, scratch=FAKE, size=1 << 30):
        return lib.falqon_block_norm_backward(p, dx, dh_out, h, *hc, y, *yc, ip, iq, dh, dy, dpost, dpre, dgate, None, scratch, size, None)

    for kw in bad:
        assert bwd(plan(tr, **kw)) == inv, kw
    assert bwd(plan(tr), dx=None) == inv and bwd(plan(tr), iq=None) == inv and bwd(plan(tr), ip=None) == inv
    assert bwd(plan(tr, flags=1), dh_out=None, dx=None) == inv
    assert bwd(plan(tr), y=None) == inv                                           # neither y nor its codes
    assert bwd(plan(tr), yc=(FAKE, FAKE)) == inv                                  # both
    assert bwd(plan(tr), y=None, yc=(FAKE, FAKE)) == inv                          # h plain, y coded
    assert bwd(plan(tr), h=None) == inv                                           # dh of a residual that was not there
    assert bwd(plan(tr), dy=FAKE) == inv                                          # dh is dy
    assert bwd(plan(tr), dh=None, dy=None, dpost=None, dpre=None, dgate=None) == inv
    assert bwd(plan(tr, gate=None)) == inv and bwd(plan(tr, post_gain=None)) == inv and bwd(plan(tr, flags=1), dx=None) == inv
    assert bwd(plan(tr), scratch=None) == fq.ERR_WORKSPACE and bwd(plan(tr), size=16) == fq.ERR_WORKSPACE
    assert bwd(plan(tr), scratch=FAKE + 4) == fq.ERR_WORKSPACE


def test_preference_refusals(fq, tr):
    inv, lib = fq.ERR_INVALID_ARG, tr.lib

    def spec(**kw):
        a = dict(rows=8, vocab=100, ld=100, pairs=2, dtype=0, kind=0, flags=0, beta=0.1, margin=0.0, label_smoothing=0.0, nll_weight=0.0)
        a.update(kw)
        return C.byref(tr.falqon_preference(*a.values()))

    def fwd(p, logits=FAKE, targets=FAKE, cu=FAKE, loss=FAKE, stats=FAKE, dlogp=FAKE, scratch=FAKE, size=1 << 30):
        return lib.falqon_preference_forward(p, logits, targets, cu, None, loss, FAKE, FAKE, FAKE, stats, dlogp, scratch, size, None)

    inf, nan = float("inf"), float("nan")
    bad = [dict(rows=0), dict(rows=1 << 26), dict(vocab=0), dict(vocab=1 << 31), dict(ld=99), dict(pairs=0), dict(dtype=3), dict(kind=3), dict(kind=-1),
           dict(flags=2), dict(beta=0.0), dict(beta=-1.0), dict(beta=nan), dict(beta=inf), dict(margin=nan), dict(margin=inf), dict(label_smoothing=-0.1),
           dict(label_smoothing=1.5), dict(label_smoothing=nan), dict(kind=1, label_smoothing=0.1), dict(nll_weight=-1.0), dict(nll_weight=nan)]
    for kw in bad:
        assert fwd(spec(**kw)) == inv, kw
        assert lib.falqon_preference_backward(spec(**kw), FAKE, FAKE, FAKE, FAKE, None, FAKE, 100, None, None) == inv, kw
    assert fwd(None) == inv and fwd(spec(), logits=None) == inv and fwd(spec(), targets=None) == inv and fwd(spec(), cu=None) == inv
    assert fwd(spec(), loss=None) == inv and fwd(spec(), stats=None) == inv and fwd(spec(), dlogp=None) == inv and fwd(spec(), stats=FAKE + 4) == inv
    assert fwd(spec(), logits=FAKE + 1) == inv and fwd(spec(dtype=1), logits=FAKE + 2) == inv
    assert fwd(spec(), scratch=None) == fq.ERR_WORKSPACE and fwd(spec(), size=100) == fq.ERR_WORKSPACE
    back = lib.falqon_preference_backward
    assert back(spec(), FAKE, FAKE, None, FAKE, None, FAKE, 100, None, None) == inv
    assert back(spec(), FAKE, FAKE, FAKE, FAKE, None, 2 * FAKE, 99, None, None) == inv             # ld_out below the vocabulary
    assert back(spec(), FAKE, FAKE, FAKE, FAKE, None, FAKE, 104, None, None) == inv                # in place with another pitch
    one = lib.falqon_sequence_logprob
    assert one(FAKE, 0, 8, 100, 100, FAKE, FAKE, 0, 0, None, FAKE, FAKE, 1 << 30, None) == inv
    assert one(FAKE, 0, 8, 100, 99, FAKE, FAKE, 2, 0, None, FAKE, FAKE, 1 << 30, None) == inv
    assert one(FAKE, 0, 8, 100, 100, FAKE, FAKE, 2, 0, None, None, FAKE, 1 << 30, None) == inv
    assert one(FAKE, 0, 8, 100, 100, FAKE, FAKE, 2, 0, None, FAKE, FAKE, 64, None) == fq.ERR_WORKSPACE
    assert lib.falqon_preference_scratch_bytes(8, 0, 0) == 0 and lib.falqon_preference_scratch_bytes(8, 100, 5) == 0


def test_scratch_sizes(tr):
    """A split row needs more scratch than a whole one, never less than one part per row."""
    size = tr.lib.falqon_preference_scratch_bytes
    assert 4096 * 8 < size(4096, 32000, 0) < 4096 * 16
    assert size(1, 32000, 0) > 8 * 8
    norm = tr.lib.falqon_block_norm_scratch_bytes
    assert norm(plan(tr, rows=4096, cols=4096, rows_per_gate=4096)) >= 2 * 4096 * 4
    assert norm(plan(tr, rows=4096, cols=64, rows_per_gate=1)) >= 4096 * 64 * 4         # a sum for every gate row


def test_the_python_calls_refuse_cpu_tensors_and_wrong_shapes(tr, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    ck = tr.Checkpoint.empty(4, 64, "cpu")
    for call in (lambda: tr.checkpoint_save(x), lambda: tr.gate_forward(x, x), lambda: tr.gate_backward(ck, ck, x), lambda: tr.block_norm_forward(x, x),
                 lambda: tr.block_norm_backward(x, x, ck, ck, torch.zeros(4), torch.zeros(4))):
        with pytest.raises(ValueError, match="current device"):
            call()
    with pytest.raises(TypeError):
        tr.block_norm_forward(x.half(), x.half())
    bad = [lambda: tr.gate_forward(x, x[:2]), lambda: tr.gate_forward(x.t(), x.t()), lambda: tr.checkpoint_save(x[:, ::2]), lambda: tr.checkpoint_save(x[:0]),
           lambda: tr.gate_backward(ck, tr.Checkpoint(ck.codes, ck.scales[:, :1]), x), lambda: tr.block_norm_forward(x, x.float()),
           lambda: tr.block_norm_forward(x, x, post_gain=torch.ones(63)), lambda: tr.block_norm_forward(x, x, pre=False, pre_gain=torch.ones(64)),
           lambda: tr.block_norm_forward(x, x, gate=torch.ones((2, 64))), lambda: tr.block_norm_forward(x, x, gate=torch.ones((2, 64)), rows_per_gate=0),
           lambda: tr.block_norm_forward(x, x, post_gain=torch.ones(64), pre_gain=torch.ones(64, dtype=torch.bfloat16)),
           lambda: tr.block_norm_backward(None, None, x, x, None, None), lambda: tr.block_norm_backward(x, x, ck, x, torch.zeros(4), torch.zeros(4)),
           lambda: tr.block_norm_backward(x, x, x, x, None, torch.zeros(4)), lambda: tr.block_norm_backward(x, x, x, x, torch.zeros(4), torch.zeros(3))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    logits, t, cu = torch.zeros((4, 10)), torch.zeros(4, dtype=torch.int64), torch.tensor([0, 2, 4])
    spec = tr.PreferenceLoss()
    for call in (lambda: tr.preference_forward(spec, logits, t.int(), cu), lambda: tr.preference_forward(spec, logits, t[:3], cu),
                 lambda: tr.preference_forward(spec, logits, t, cu[:2]), lambda: tr.preference_forward(spec, logits.t(), t, cu),
                 lambda: tr.preference_forward(spec._replace(kind="dpo"), logits, t, cu), lambda: tr.preference_forward(spec, logits, t, cu, torch.zeros(1)),
                 lambda: tr.sequence_logprob(logits, t, cu[:1]), lambda: tr.preference_forward(spec, logits, t, cu)):
        with pytest.raises(ValueError):
            call()
