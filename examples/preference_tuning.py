"""Preference tuning of a small decoder-shaped model with melded FP8-LoRA layers: every step of it runs in the library's kernels.

Per block (hidden width H, MLP width F; every linear is a melded layer with its own adapter):

    q, k, v = L_q(x), L_k(x), L_v(x);  a = (q + k + v) / sqrt(3)                 a stand-in for the attention's mixing
    h, x = block norm(h, L_o(a))            norm after the block, its gate, the residual scale, norm before the MLP
    z = silu(L_gate(x)) * L_up(x)
    h, x = block norm(h, L_down(z))

What the backward needs is kept in 8 bits: the inputs of each block norm and of each gated product.  After the last block,
logits = L_head(x) and the preference loss of pairs of sequences against the log-probabilities of the same model before tuning.
The adapters' gradients go to their DeltaBuffers (one batched proxy update per step), the gains' and gates' to plain SGD.

    python examples/preference_tuning.py [--steps 12]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2510_24061_b200 import binding as fq  # noqa: E402
from paper_2510_24061_b200 import stack, synth  # noqa: E402
from paper_2510_24061_b200 import training as tr  # noqa: E402

INV_SQRT3 = 1.0 / math.sqrt(3.0)


class Junction:
    """The norm after a block and the norm before the next one, with the block's gate (one row for all tokens)."""

    def __init__(self, H: int, device, post: bool = True):
        one = lambda v: torch.full((H,), v, dtype=torch.float32, device=device)  # noqa: E731
        self.kw = dict(pre_gain=one(1.0), res_scale=1.0)
        if post:
            self.kw |= dict(post_gain=one(1.0), gate=one(0.5))
        else:
            self.kw |= dict(post=False)

    def forward(self, h, y, amax):
        out = tr.block_norm_forward(h, y, save=True, amax_x=amax, **self.kw)
        self.saved = out.saved_h, out.saved_y, out.inv_post, out.inv_pre
        return out.h_out, out.x

    def backward(self, dx, dh_out, amax_dy=None, lr: float = 0.0):
        saved_h, saved_y, inv_post, inv_pre = self.saved
        g = tr.block_norm_backward(dx, dh_out, saved_h, saved_y, inv_post, inv_pre, amax_dy=amax_dy, **self.kw)
        for name, grad in (("post_gain", g.dpost_gain), ("pre_gain", g.dpre_gain), ("gate", g.dgate)):
            if grad is not None:
                self.kw[name] -= lr * grad.view_as(self.kw[name])
        return g.dh, g.dy


class Model:
    def __init__(self, blocks: int, H: int, F: int, vocab: int, T: int, r: int, seed: int, device):
        self.T, self.device, self.layers, self.order = T, device, {}, []
        shapes = {"q": (H, H), "k": (H, H), "v": (H, H), "o": (H, H), "gate": (F, H), "up": (F, H), "down": (H, F)}
        for name, (m, n) in [((b, p), s) for b in range(blocks) for p, s in shapes.items()] + [(("head", "head"), (vocab, H))]:
            mat = len(self.order)
            W = (synth.backbone(seed, mat, m, n, device).float() * (2.0 if name[0] != "head" else 4.0)).to(torch.bfloat16)
            self.layers[name] = fq.setup_layer(W, synth.adapter_a(seed, mat, r, n, device), None, 1.0)
            self.order.append(name)
        self.blocks = blocks
        self.embedding = synth.normal_bf16(seed, 90001, (vocab, H), 1.0, device)
        self.first = Junction(H, device, post=False)
        self.norms = [(Junction(H, device), Junction(H, device)) for _ in range(blocks)]
        self.kept, self.dB = {}, {}

    def _linear(self, name, x, amax):
        layer = self.layers[name]
        Y, OA, amax_oa, _ = fq.melded_forward(layer, x, amax_x=amax)
        self.kept[name] = OA, amax_oa
        return Y

    def _linear_grad(self, name, dY, amax=None):
        OA, amax_oa = self.kept[name]
        dX, self.dB[name], _ = fq.melded_backward(self.layers[name], dY, OA, amax_oa, amax_dy=amax)
        return dX

    def _words(self, n):
        """Zeroed words for the absmax that a producing kernel hands to the layer that takes its result."""
        return torch.zeros(n, dtype=torch.float32, device=self.device).split(1)

    def forward(self, tokens: torch.Tensor) -> torch.Tensor:
        am = self._words(1 + 4 * self.blocks)
        h, x = self.first.forward(None, self.embedding[tokens], am[0])
        amax_x = am[0]
        self.mlp = []
        for b in range(self.blocks):
            a1, a2, a3, a4 = am[1 + 4 * b:5 + 4 * b]
            q, k, v = (self._linear((b, p), x, amax_x) for p in "qkv")
            stack.combine(q, q, INV_SQRT3, k, INV_SQRT3, v, INV_SQRT3, amax=a1)
            h, x = self.norms[b][0].forward(h, self._linear((b, "o"), q, a1), a2)
            z, kept_g, kept_u = tr.gate_forward(self._linear((b, "gate"), x, a2), self._linear((b, "up"), x, a2), amax=a3)
            self.mlp.append((kept_g, kept_u))
            h, x = self.norms[b][1].forward(h, self._linear((b, "down"), z, a3), a4)
            amax_x = a4
        return self._linear(("head", "head"), x, amax_x)

    def backward(self, dlogits: torch.Tensor, amax, norm_lr: float):
        am = self._words(5 * self.blocks)
        dx, dh = self._linear_grad(("head", "head"), dlogits, amax), None
        for b in reversed(range(self.blocks)):
            a1, a2, a3, a4, a5 = am[5 * b:5 * b + 5]
            dh, dy = self.norms[b][1].backward(dx, dh, a1, norm_lr)
            dz = self._linear_grad((b, "down"), dy, a1)
            dg, du = tr.gate_backward(*self.mlp[b], dz, amax_dg=a2, amax_du=a3)
            dx = stack.combine(dz.new_empty(dh.shape), self._linear_grad((b, "gate"), dg, a2), 1.0, self._linear_grad((b, "up"), du, a3), 1.0)
            dh, dy = self.norms[b][0].backward(dx, dh, a4, norm_lr)
            da = self._linear_grad((b, "o"), dy, a4)
            stack.combine(da, da, INV_SQRT3, amax=a5)
            dq, dk, dv = (self._linear_grad((b, p), da, a5) for p in "qkv")
            dx = stack.combine(dq, dq, 1.0, dk, 1.0, dv, 1.0)
        self.first.backward(dx, dh, None, norm_lr)

    def update(self, lr: float, k: int):
        for i in range(0, len(self.order), 8):
            names = self.order[i:i + 8]
            fq.proxy_update_batched([self.layers[n] for n in names], [self.dB[n] for n in names], lr,
                                    [min(k, self.layers[n].m) for n in names])


def batch(pairs: int, length: int, prompt: int, vocab: int, seed: int, device):
    """Pairs of token sequences that share a prompt, packed; a row's target is the token after it, and prompt rows have none."""
    gen = torch.Generator().manual_seed(seed)
    seqs, targets, bounds = [], [], [0]
    for _ in range(pairs):
        head = torch.randint(0, vocab, (prompt,), generator=gen)
        for _ in range(2):
            t = torch.cat([head, torch.randint(0, vocab, (length - prompt + int(torch.randint(0, 5, (1,), generator=gen)),), generator=gen)])
            y = torch.cat([t[1:], torch.tensor([-100])])
            y[:prompt - 1] = -100
            seqs.append(t)
            targets.append(y)
            bounds.append(bounds[-1] + len(t))
    return torch.cat(seqs).to(device), torch.cat(targets).to(device), torch.tensor(bounds, device=device)


def train(steps: int = 12, blocks: int = 2, H: int = 256, F: int = 512, vocab: int = 1008, pairs: int = 4, lr: float = 0.3, norm_lr: float = 0.01, seed: int = 0):
    """Returns the losses of the steps, and the share of pairs in which the chosen sequence gained more, after the last."""
    device = torch.device("cuda")
    tokens, targets, cu = batch(pairs, 24, 8, vocab, seed, device)
    model = Model(blocks, H, F, vocab, tokens.numel(), 16, seed, device)
    ref, _ = tr.sequence_logprob(model.forward(tokens), targets, cu)         # the model before tuning is the reference
    spec = tr.PreferenceLoss(beta=0.5)
    losses = []
    for _ in range(steps):
        logits = model.forward(tokens)
        out = tr.preference_forward(spec, logits, targets, cu, ref)
        amax = torch.zeros(1, device=device)
        model.backward(tr.preference_backward(logits, targets, out, dlogits=logits, amax=amax), amax, norm_lr)
        model.update(lr, k=H)
        losses.append(out.loss)
    gained = out.seq_logp - ref
    assert fq.last_device_status() == fq.OK
    return [float(v) for v in losses], float((gained[0::2] > gained[1::2]).float().mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=12)
    losses, right = train(ap.parse_args().steps)
    for i, v in enumerate(losses):
        print(f"step {i:3d}  loss {v:.5f}")
    print(f"chosen sequence ahead in {100 * right:.0f} % of the pairs")
