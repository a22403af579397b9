"""Every buffer that a call of include/falqon_train.h may write lies between margins of a pattern: none is touched, at sizes whose last
vectors, spans, rows, runs and tiles are partial."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu

MARGIN = 4096


class Fenced:
    """A tensor between two margins, in one allocation."""

    def __init__(self, shape, dtype):
        n = 1
        for s in shape:
            n *= s
        self.bytes = n * torch.empty(0, dtype=dtype).element_size()
        room = (self.bytes + 15) // 16 * 16
        self.store = torch.full((2 * MARGIN + room,), 0xA5, dtype=torch.uint8, device="cuda")
        self.t = self.store[MARGIN:MARGIN + self.bytes].view(dtype).view(shape)
        self.p = self.t.data_ptr()

    def check(self, what):
        assert (self.store[:MARGIN] == 0xA5).all() and (self.store[MARGIN + self.bytes:] == 0xA5).all(), f"margins of {what} written"


@pytest.fixture(scope="module")
def tr():
    from paper_2510_24061_b200 import training
    return training


def fence(**shapes):
    return {k: Fenced(*v) for k, v in shapes.items()}


def finish(call, out, **what):
    torch.cuda.synchronize()
    assert call == 0, what
    for k, f in out.items():
        f.check(f"{k} at {what}")


SIZES = [(1, 1), (1, 7), (3, 40), (5, 1011), (2, 4095), (9, 512), (1, 4096), (33, 1000), (3, 5136), (150, 97), (2, 8192), (4, 11008), (3, 16383)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_gate_and_checkpoints(tr, rows, cols, dtype):
    code, nb = (0 if dtype == torch.bfloat16 else 1), -(-cols // 32)
    g, u, dz = (torch.randn((rows, cols), device="cuda").to(dtype) for _ in range(3))
    u8 = torch.uint8
    out = fence(z=((rows, cols), dtype), gc=((rows, cols), u8), gs=((rows, nb), u8), uc=((rows, cols), u8), us=((rows, nb), u8), amax=((1,), torch.float32))
    finish(tr.lib.falqon_gate_forward(g.data_ptr(), u.data_ptr(), code, rows, cols, out["z"].p, out["gc"].p, out["gs"].p, out["uc"].p, out["us"].p, out["amax"].p, None),
           out, rows=rows, cols=cols)
    back = fence(dg=((rows, cols), dtype), du=((rows, cols), dtype))
    finish(tr.lib.falqon_gate_backward(out["gc"].p, out["gs"].p, out["uc"].p, out["us"].p, dz.data_ptr(), code, rows, cols, back["dg"].p, back["du"].p, None, None, None),
           back, rows=rows, cols=cols)
    one = fence(c=((rows, cols), u8), s=((rows, nb), u8), x=((rows, cols), dtype))
    finish(tr.lib.falqon_checkpoint_save(g.data_ptr(), code, rows, cols, one["c"].p, one["s"].p, None), one, rows=rows, cols=cols)
    finish(tr.lib.falqon_checkpoint_load(one["c"].p, one["s"].p, rows, cols, one["x"].p, code, None), one, rows=rows, cols=cols)
    assert torch.equal(one["c"].t, out["gc"].t) and torch.equal(one["s"].t, out["gs"].t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_block_norm(tr, rows, cols, dtype):
    code, nb, rpg = (0 if dtype == torch.bfloat16 else 1), -(-cols // 32), max(1, rows // 3)
    gates = -(-rows // rpg)
    h, y, dx, dh_out = (torch.randn((rows, cols), device="cuda").to(dtype) for _ in range(4))
    w1, w2, gate = (torch.randn(n, device="cuda") for n in (cols, cols, gates * cols))
    plan = tr.falqon_block_norm(rows, cols, rpg, code, 1, 3, 0.5, 0.0, 1e-6, w1.data_ptr(), w2.data_ptr(), gate.data_ptr())
    u8, f32 = torch.uint8, torch.float32
    out = fence(h_out=((rows, cols), dtype), x=((rows, cols), dtype), ip=((rows,), f32), iq=((rows,), f32), hc=((rows, cols), u8), hs=((rows, nb), u8),
                yc=((rows, cols), u8), ys=((rows, nb), u8), amax=((1,), f32))
    o = {k: v.p for k, v in out.items()}
    finish(tr.lib.falqon_block_norm_forward(C.byref(plan), h.data_ptr(), y.data_ptr(), o["h_out"], o["x"], o["ip"], o["iq"], o["hc"], o["hs"], o["yc"], o["ys"], o["amax"], None),
           out, rows=rows, cols=cols)
    size = tr.lib.falqon_block_norm_scratch_bytes(C.byref(plan))
    for coded in (True, False):
        back = fence(dh=((rows, cols), dtype), dy=((rows, cols), dtype), d1=((cols,), f32), d2=((cols,), f32), dg=((gates, cols), f32), scratch=((size,), u8))
        b = {k: v.p for k, v in back.items()}
        saved = (None, o["hc"], o["hs"], None, o["yc"], o["ys"]) if coded else (h.data_ptr(), None, None, y.data_ptr(), None, None)
        finish(tr.lib.falqon_block_norm_backward(C.byref(plan), dx.data_ptr(), dh_out.data_ptr(), *saved, o["ip"], o["iq"], b["dh"], b["dy"], b["d1"], b["d2"], b["dg"],
                                                 None, b["scratch"], size, None), back, rows=rows, cols=cols, coded=coded)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (2, 9), (7, 1001), (40, 32003), (3, 50001), (130, 515), (2, 131072)])
def test_preference(tr, rows, vocab, dtype):
    code, pairs = (0 if dtype == torch.bfloat16 else 1), max(1, rows // 8)
    logits = torch.randn((rows, vocab), device="cuda").to(dtype)
    targets = torch.randint(0, vocab, (rows,), device="cuda")
    targets[::3] = -1
    cu = torch.linspace(0, rows, 2 * pairs + 1).long().cuda()
    f32 = torch.float32
    size = tr.lib.falqon_preference_scratch_bytes(rows, vocab, code)
    out = fence(loss=((1,), f32), pair=((pairs,), f32), seq=((2 * pairs,), f32), logp=((rows,), f32), stats=((rows, 2), f32), dlogp=((rows,), f32),
                scratch=((size,), torch.uint8), dlogits=((rows, vocab), dtype), seq2=((2 * pairs,), f32), logp2=((rows,), f32))
    o = {k: v.p for k, v in out.items()}
    plan = tr.falqon_preference(rows, vocab, vocab, pairs, code, 0, 0, 0.1, 0.0, 0.0, 0.0)
    finish(tr.lib.falqon_preference_forward(C.byref(plan), logits.data_ptr(), targets.data_ptr(), cu.data_ptr(), None, o["loss"], o["pair"], o["seq"], o["logp"], o["stats"],
                                            o["dlogp"], o["scratch"], size, None), out, rows=rows, vocab=vocab)
    finish(tr.lib.falqon_preference_backward(C.byref(plan), logits.data_ptr(), targets.data_ptr(), o["stats"], o["dlogp"], None, o["dlogits"], vocab, None, None),
           out, rows=rows, vocab=vocab)
    finish(tr.lib.falqon_sequence_logprob(logits.data_ptr(), code, rows, vocab, vocab, targets.data_ptr(), cu.data_ptr(), 2 * pairs, 0, o["logp2"], o["seq2"], o["scratch"],
                                          size, None), out, rows=rows, vocab=vocab)
    assert torch.equal(out["seq"].t, out["seq2"].t) and torch.equal(out["logp"].t, out["logp2"].t)
