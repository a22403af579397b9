"""Limits and refusals of include/falqon_train.h that need no GPU: what would overflow, or leave a wrong result, is refused before any launch."""
import ctypes as C
import os
import re

import pytest

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


def plan(tr, **kw):
    a = dict(rows=8, cols=64, rows_per_gate=8, dtype=0, gain_dtype=1, flags=3, res_scale=1.0, gain_offset=0.0, eps=1e-6, post_gain=FAKE,
             pre_gain=FAKE, gate=FAKE)
    a.update(kw)
    return C.byref(tr.falqon_block_norm(*a.values()))


def test_rows_beyond_what_the_kernels_can_count_are_refused(fq, tr):
    """Row numbers are 32 bits and kernels look up to 4 stages of 16 rows ahead: row + 64 has to stay below 2^31.  The largest count that
    is taken is asked of the scratch size only, which launches nothing."""
    header = open(os.path.join(ROOT, "include", "falqon_train.h")).read()
    limit = int(re.search(r"#define FALQON_NORM_MAX_ROWS (\d+)", header).group(1))
    assert limit == tr.NORM_MAX_ROWS and limit + 64 < 1 << 31
    for rows in (limit + 1, (1 << 31) - 1, 1 << 31):
        p = plan(tr, rows=rows, cols=1, rows_per_gate=rows)
        assert tr.lib.falqon_block_norm_scratch_bytes(p) == 0
        assert tr.lib.falqon_block_norm_forward(p, FAKE, FAKE, FAKE, 2 * FAKE, FAKE, FAKE, *(None,) * 6) == fq.ERR_INVALID_ARG
        assert tr.lib.falqon_block_norm_backward(p, FAKE, FAKE, FAKE, None, None, FAKE, None, None, FAKE, FAKE, FAKE, 2 * FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 40,
                                                 None) == fq.ERR_INVALID_ARG
    assert tr.lib.falqon_block_norm_scratch_bytes(plan(tr, rows=limit, cols=1, rows_per_gate=limit)) > 0


def test_two_results_in_one_buffer_are_refused(fq, tr):
    """h_out and x written to the same place would leave a mixture of the two: refused, as dh = dy is in the backward."""
    fwd = tr.lib.falqon_block_norm_forward
    assert fwd(plan(tr), FAKE, 2 * FAKE, 3 * FAKE, 3 * FAKE, FAKE, FAKE, *(None,) * 6) == fq.ERR_INVALID_ARG
    assert fwd(plan(tr), FAKE, 2 * FAKE, FAKE, FAKE, FAKE, FAKE, *(None,) * 6) == fq.ERR_INVALID_ARG           # h_out in place of h, and x there too


def test_the_stream_is_found_without_torchs_private_entry(tr, monkeypatch):
    """The handle comes from a private entry of torch where it has one, else from the public stream object."""
    class Stream:
        cuda_stream = 0x5EED

    monkeypatch.setattr(tr.torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(tr.torch.cuda, "current_stream", lambda dev: Stream())
    monkeypatch.setattr(tr, "_raw_stream", None)
    assert tr._on_device() == 0x5EED


def test_choices_of_results_are_checked(tr, monkeypatch):
    monkeypatch.setattr(tr.torch.cuda, "current_device", lambda: 0)
    x, inv = tr.torch.zeros((4, 64)), tr.torch.zeros(4)
    one = tr.torch.zeros(1)
    for call in (lambda: tr.block_norm_forward(x, x, pre=False, need_h_out=False), lambda: tr.block_norm_forward(x, x, h_out=x.clone(), need_h_out=False),
                 lambda: tr.block_norm_backward(x, x, x, x, inv, inv, need_gains=("gain",)), lambda: tr.block_norm_backward(x, x, x, x, inv, inv, need_gains="gate"),
                 lambda: tr.block_norm_backward(x, x, x, x, inv, inv, need_dy=False, dy=x.clone()),
                 lambda: tr.block_norm_backward(x, x, x, x, inv, inv, need_dy=False, amax_dy=one)):
        with pytest.raises(ValueError, match="wanted|need_gains|without h_out"):
            call()
