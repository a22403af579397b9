"""The operators that stand between and behind the melded layers in a fine-tuning step, as cases that can be timed and checked:

* ``norm``: the norms after and before a block, fused with the block's gate and the residual scale, forward and backward;
* ``gate``: the SiLU-gated product of the MLP, whose inputs are kept for the backward as 8-bit checkpoints, forward and backward;
* ``pref``: the preference loss of paired sequences (log ratios against a reference), alone and with the gradient of the logits.

``run`` computes them in plain torch operations in 32 bits, or, where ``own`` is set, by the package's calls.
"""
from __future__ import annotations

import random

import torch

own = False

EPS = 1e-6
BETA, SMOOTHING, NLL_WEIGHT = 0.1, 0.05, 0.2
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32          # values that share a scale in an 8-bit checkpoint


# ---------------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a single token through the norms around a block: serving, where the call's latency is all that counts
        dict(name="norm fwd, one token", op="norm", way="fwd", rows=1, cols=4096, dtype="bf16", saved="none", gates=1),
        # a step of 4096 tokens through a 7B-shaped block, the norm's inputs kept in 8 bits for the backward
        dict(name="norm fwd, 7B, checkpoints", op="norm", way="fwd", rows=4096, cols=4096, dtype="bf16", saved="codes", gates=1),
        # its backward, from the checkpoints
        dict(name="norm bwd, 7B, checkpoints", op="norm", way="bwd", rows=4096, cols=4096, dtype="bf16", saved="codes", gates=1),
        # the 13B width and 8192 tokens, inputs kept as they are, a gate of its own for each of 16 sequences
        dict(name="norm bwd, 13B, gates", op="norm", way="bwd", rows=8192, cols=5120, dtype="bf16", saved="plain", gates=16),
        # an odd width in 32 bits, as a small model under test has it
        dict(name="norm bwd, odd width, f32", op="norm", way="bwd", rows=613, cols=1011, dtype="f32", saved="codes", gates=5),
        # a single token through the gated MLP, checkpoints kept
        dict(name="gate fwd, one token", op="gate", way="fwd", rows=1, cols=11008, dtype="bf16"),
        # the 7B MLP in a step of 4096 tokens
        dict(name="gate fwd, 7B", op="gate", way="fwd", rows=4096, cols=11008, dtype="bf16"),
        # the 13B MLP's backward from its checkpoints, 8192 tokens
        dict(name="gate bwd, 13B", op="gate", way="bwd", rows=8192, cols=13824, dtype="bf16"),
        # one short pair: the step of a small batch, few rows and a long vocabulary
        dict(name="pref step, one short pair", op="pref", way="step", rows=49, vocab=32000, pairs=1, dtype="bf16", kind="sigmoid", average=False),
        # a vocabulary of odd length in 32 bits, length-normalised
        dict(name="pref step, odd vocab, f32", op="pref", way="step", rows=701, vocab=32003, pairs=3, dtype="f32", kind="ipo", average=True),
        # evaluation: the loss and the sequences' log-probabilities alone
        dict(name="pref fwd, evaluation", op="pref", way="fwd", rows=4096, vocab=32000, pairs=8, dtype="bf16", kind="sigmoid", average=False),
        # a whole training batch: 16384 tokens of 16 pairs
        dict(name="pref step, batch", op="pref", way="step", rows=16384, vocab=32000, pairs=16, dtype="bf16", kind="sigmoid", average=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(torch.log2(torch.tensor(float(lo))).item(), torch.log2(torch.tensor(float(hi))).item())))


def draw(rng: random.Random):
    op = rng.choice(["norm", "gate", "pref"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "pref":
        rows, vocab = _log_int(rng, 4, 16384), _log_int(rng, 1000, 130000)
        rows = max(4, min(rows, 16384 * 32000 * 2 // (vocab * (4 if dtype == "f32" else 2))))
        return dict(op=op, way=rng.choice(["step", "step", "fwd"]), rows=rows, vocab=vocab, pairs=rng.randint(1, max(1, min(16, rows // 4))),
                    dtype=dtype, kind=rng.choice(["sigmoid", "hinge", "ipo"]), average=rng.random() < 0.5)
    cols = _log_int(rng, 64, 16384) if op == "norm" else _log_int(rng, 64, 28672)
    if rng.random() < 0.7:      # widths are mostly multiples of a tile; the others stay as they come
        cols = max(64, cols // 64 * 64)
    rows = min(_log_int(rng, 1, 16384), (1 << 27) // cols)
    if op == "gate":
        return dict(op=op, way=rng.choice(["fwd", "bwd"]), rows=rows, cols=cols, dtype=dtype)
    way = rng.choice(["fwd", "bwd"])
    return dict(op=op, way=way, rows=rows, cols=cols, dtype=dtype, saved=rng.choice(["codes", "plain"] if way == "bwd" else ["codes", "none"]),
                gates=rng.choice([1, 1, min(rows, rng.randint(2, 32))]))


def _rows_per_gate(case):
    return -(-case["rows"] // case["gates"])


def _gates(case):
    return -(-case["rows"] // _rows_per_gate(case))


def _lengths(case):
    """Rows of each of the 2 x pairs sequences, and how many at the head of each are prompt (not counted): ragged, by the case alone."""
    rng = random.Random(case["rows"] * 1000003 + case["pairs"])
    n = 2 * case["pairs"]
    weight = [rng.uniform(0.5, 1.5) for _ in range(n)]
    cuts = [0]
    for i in range(n):
        cuts.append(round(case["rows"] * sum(weight[:i + 1]) / sum(weight)))
    lens = [b - a for a, b in zip(cuts, cuts[1:])]
    return lens, [l // 4 for l in lens]


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    code = 1 + 1 / BLOCK
    if case["op"] == "pref":
        lens, prompt = _lengths(case)
        counted = sum(lens) - sum(prompt)
        read, every = counted * case["vocab"], case["rows"] * case["vocab"]
        small = case["rows"] * (8 + 4)
        if case["way"] == "fwd":
            return {"bytes": read * size + small, "flops": 4 * read}
        return {"bytes": read * size + every * size + small, "flops": 8 * read}
    n = case["rows"] * case["cols"]
    if case["op"] == "gate":
        return {"bytes": n * (3 * size + 2 * code), "flops": n * (12 if case["way"] == "fwd" else 20)}
    gains = case["cols"] * 4 * (2 + _gates(case)) + case["rows"] * 8
    if case["way"] == "fwd":
        return {"bytes": n * (4 * size + (2 * code if case["saved"] == "codes" else 0)) + gains, "flops": 12 * n}
    return {"bytes": n * (4 * size + 2 * (code if case["saved"] == "codes" else size)) + 2 * gains, "flops": 30 * n}


# ---------------------------------------------------------------------------------------------------------------- the inputs
def _normal(gen, shape, scale, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _random_codes(gen, rows, cols, scale):
    """A checkpoint of normal values, in torch: codes and scale bytes."""
    x = torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.float32).mul_(scale)
    codes, scales = _encode(x)
    return codes.view(torch.uint8), scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "pref":
        rows, vocab = case["rows"], case["vocab"]
        lens, prompt = _lengths(case)
        logits = torch.randn((rows, vocab), generator=gen, device="cuda", dtype=dt).mul_(2.0)
        targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        likely = torch.arange(rows, device="cuda")
        logits[likely, targets] += 9.0          # a model that has learnt something gives the target a few per cent
        counted = torch.cat([torch.arange(l) >= p for l, p in zip(lens, prompt)]).cuda()
        # what a reference model says of these sequences: close to the policy's own (the logits are N(0, 2): lse = ln vocab + 2)
        near = torch.where(counted, logits[likely, targets].float() - (float(torch.log(torch.tensor(float(vocab)))) + 2.0), torch.zeros(rows, device="cuda"))
        cu = torch.tensor([0] + lens).cumsum(0)
        seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).cuda()
        ref = (near * (seq == torch.arange(len(lens), device="cuda")[:, None])).sum(1)
        if case["average"]:
            ref = ref / torch.tensor([max(1, l - p) for l, p in zip(lens, prompt)], device="cuda")
            ref += torch.randn(ref.shape, generator=gen, device="cuda") * 0.5
        else:
            ref += torch.randn(ref.shape, generator=gen, device="cuda") * 10.0
        s |= dict(logits=logits, targets=torch.where(counted, targets, -100), cu=cu.cuda(), ref=ref)
        return s
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "gate":
        if case["way"] == "fwd":
            s |= dict(g=_normal(gen, (rows, cols), 1.5, dt), u=_normal(gen, (rows, cols), 1.0, dt))
        else:
            s |= dict(g=_random_codes(gen, rows, cols, 1.5), u=_random_codes(gen, rows, cols, 1.0), dz=_normal(gen, (rows, cols), 1e-2, dt))
        return s
    s |= dict(post_gain=_normal(gen, (cols,), 0.1, torch.float32).add_(1.0), pre_gain=_normal(gen, (cols,), 0.1, torch.float32).add_(1.0),
              gate=_normal(gen, (_gates(case), cols), 0.2, torch.float32).add_(0.5), res_scale=0.9)
    if case["way"] == "fwd":
        s |= dict(h=_normal(gen, (rows, cols), 2.0, dt), y=_normal(gen, (rows, cols), 0.7, dt))
        return s
    if case["saved"] == "codes":
        s |= dict(h=_random_codes(gen, rows, cols, 2.0), y=_random_codes(gen, rows, cols, 0.7))
    else:
        s |= dict(h=_normal(gen, (rows, cols), 2.0, dt), y=_normal(gen, (rows, cols), 0.7, dt))
    # the inverse root mean squares as the forward leaves them, of the tensors before they were rounded to 8 bits
    s |= dict(inv_post=1.0 / (0.7 + 0.02 * torch.randn(rows, generator=gen, device="cuda")), inv_pre=1.0 / (1.9 + 0.05 * torch.randn(rows, generator=gen, device="cuda")),
              dx=_normal(gen, (rows, cols), 1e-2, dt), dh_out=_normal(gen, (rows, cols), 1e-2, dt))
    return s


# ---------------------------------------------------------------------------------------------------------------- the plain forms
def _encode(x):
    """E4M3 codes of 32-bit x [rows, cols] and the exponent byte of each block of 32 values of a row: the smallest power of two that brings
    the block's largest value to 448 or below."""
    rows, cols = x.shape
    pad = -cols % BLOCK
    blocks = torch.nn.functional.pad(x, (0, pad)).view(rows, -1, BLOCK)
    mantissa, exponent = torch.frexp(blocks.abs().amax(2))              # amax = mantissa * 2^exponent, 0.5 <= mantissa < 1
    e = torch.clamp(exponent - 9 + (mantissa > 0.875) + 127, min=0)
    scaled = torch.ldexp(blocks, (127 - e)[:, :, None]).view(rows, -1)[:, :cols]
    return scaled.to(torch.float8_e4m3fn), e.to(torch.uint8)


def _decode(codes, scales):
    rows, cols = codes.shape
    e = scales.to(torch.int32) - 127
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), e.repeat_interleave(BLOCK, 1)[:, :cols])


def _plain_norm(s, case):
    dt = DTYPES[case["dtype"]]
    per_row = torch.arange(case["rows"], device="cuda") // _rows_per_gate(case)
    wpost, wpre, scale = s["post_gain"], s["pre_gain"], s["res_scale"]
    gate = s["gate"][per_row]
    if case["way"] == "fwd":
        h, y = s["h"].float(), s["y"].float()
        ip = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
        H = scale * h + gate * (y * ip * wpost)
        iq = torch.rsqrt((H * H).mean(1, keepdim=True) + EPS)
        out = dict(h_out=H.to(dt), x=(H * iq * wpre).to(dt), inv_post=ip[:, 0], inv_pre=iq[:, 0])
        if case["saved"] == "codes":
            out["h_codes"], out["h_scales"] = _encode(h)
            out["y_codes"], out["y_scales"] = _encode(y)
        return out
    h, y = (_decode(*s[k]) if case["saved"] == "codes" else s[k].float() for k in ("h", "y"))
    ip, iq = s["inv_post"][:, None], s["inv_pre"][:, None]
    dx, dh_out = s["dx"].float(), s["dh_out"].float()
    yh = y * ip
    xh = (scale * h + gate * (yh * wpost)) * iq
    a = dx * wpre
    d = dh_out + iq * (a - xh * (a * xh).mean(1, keepdim=True))
    b = gate * d * wpost
    dy = ip * (b - yh * (b * yh).mean(1, keepdim=True))
    of_gate = (d * yh * wpost)
    pad = _gates(case) * _rows_per_gate(case) - case["rows"]
    dgate = torch.nn.functional.pad(of_gate, (0, 0, 0, pad)).view(_gates(case), -1, case["cols"]).sum(1)
    return dict(dh=(scale * d).to(dt), dy=dy.to(dt), dpost_gain=(gate * d * yh).sum(0), dpre_gain=(dx * xh).sum(0), dgate=dgate)


def _plain_gate(s, case):
    dt = DTYPES[case["dtype"]]
    if case["way"] == "fwd":
        g, u = s["g"].float(), s["u"].float()
        gc, gs = _encode(g)
        uc, us = _encode(u)
        return dict(z=(g / (1.0 + torch.exp(-g)) * u).to(dt), g_codes=gc, g_scales=gs, u_codes=uc, u_scales=us)
    g, u, dz = _decode(*s["g"]), _decode(*s["u"]), s["dz"].float()
    sg = 1.0 / (1.0 + torch.exp(-g))
    return dict(dg=(dz * u * sg * (1.0 + g * (1.0 - sg))).to(dt), du=(dz * g * sg).to(dt))


def _log_sigmoid(d):
    return torch.clamp(d, max=0.0) - torch.log1p(torch.exp(-d.abs()))


def _plain_pref(s, case):
    dt, pairs = DTYPES[case["dtype"]], case["pairs"]
    x, targets = s["logits"].float(), s["targets"]
    counted = targets >= 0
    top = x.max(1, keepdim=True).values
    ex = torch.exp(x - top)
    total = ex.sum(1, keepdim=True)
    at = torch.clamp(targets, min=0)[:, None]
    logp = torch.where(counted, (x.gather(1, at) - top - torch.log(total))[:, 0], 0.0)
    member = (torch.arange(x.shape[0], device="cuda") >= s["cu"][:-1, None]) & (torch.arange(x.shape[0], device="cuda") < s["cu"][1:, None])
    count = (member & counted).sum(1).clamp(min=1).float()
    total_logp = (member * logp).sum(1)
    seq = total_logp / count if case["average"] else total_logp
    ratio = seq - s["ref"]
    u = ratio[0::2] - ratio[1::2]
    d = BETA * u
    if case["kind"] == "sigmoid":
        loss = -(1 - SMOOTHING) * _log_sigmoid(d) - SMOOTHING * _log_sigmoid(-d)
        du = BETA * (-(1 - SMOOTHING) / (1 + torch.exp(d)) + SMOOTHING / (1 + torch.exp(-d)))
    elif case["kind"] == "hinge":
        loss, du = torch.clamp(1 - d, min=0.0), torch.where(d < 1, -BETA, 0.0)
    else:
        loss, du = (u - 1 / (2 * BETA)) ** 2, 2 * (u - 1 / (2 * BETA))
    loss = loss - NLL_WEIGHT * total_logp[0::2] / count[0::2]
    out = dict(loss=loss.mean(), pair_loss=loss, seq_logp=seq, logp=logp)
    if case["way"] == "fwd":
        return out
    of_seq = torch.stack((du, -du), 1).view(-1) / pairs
    if case["average"]:
        of_seq = of_seq / count
    of_nll = torch.stack((NLL_WEIGHT / count[0::2] / pairs, torch.zeros_like(du)), 1).view(-1)
    coef = torch.where(counted, (member * (of_seq - of_nll)[:, None]).sum(0), 0.0)[:, None]
    grad = ex.mul_(-coef / total)
    grad.scatter_add_(1, at, coef)
    out["dlogits"] = torch.where(counted[:, None], grad, 0.0).to(dt)
    return out


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if not own:
        return {"norm": _plain_norm, "gate": _plain_gate, "pref": _plain_pref}[case["op"]](state, case)
    from paper_2510_24061_b200 import training as tr
    f8 = torch.float8_e4m3fn
    s = state
    if case["op"] == "norm":
        norms = dict(post_gain=s["post_gain"], pre_gain=s["pre_gain"], gate=s["gate"], rows_per_gate=_rows_per_gate(case), res_scale=s["res_scale"], eps=EPS)
        if case["way"] == "fwd":
            r = tr.block_norm_forward(s["h"], s["y"], save=case["saved"] == "codes", **norms)
            out = dict(h_out=r.h_out, x=r.x, inv_post=r.inv_post, inv_pre=r.inv_pre)
            if case["saved"] == "codes":
                out |= dict(h_codes=r.saved_h.codes.view(f8), h_scales=r.saved_h.scales, y_codes=r.saved_y.codes.view(f8), y_scales=r.saved_y.scales)
            return out
        h, y = (tr.Checkpoint(*s[k]) if case["saved"] == "codes" else s[k] for k in ("h", "y"))
        g = tr.block_norm_backward(s["dx"], s["dh_out"], h, y, s["inv_post"], s["inv_pre"], **norms)
        return dict(dh=g.dh, dy=g.dy, dpost_gain=g.dpost_gain, dpre_gain=g.dpre_gain, dgate=g.dgate)
    if case["op"] == "gate":
        if case["way"] == "fwd":
            z, g, u = tr.gate_forward(s["g"], s["u"])
            return dict(z=z, g_codes=g.codes.view(f8), g_scales=g.scales, u_codes=u.codes.view(f8), u_scales=u.scales)
        dg, du = tr.gate_backward(tr.Checkpoint(*s["g"]), tr.Checkpoint(*s["u"]), s["dz"])
        return dict(dg=dg, du=du)
    loss = tr.PreferenceLoss(kind=case["kind"], beta=BETA, label_smoothing=SMOOTHING if case["kind"] == "sigmoid" else 0.0, average=case["average"], nll_weight=NLL_WEIGHT)
    r = tr.preference_forward(loss, s["logits"], s["targets"], s["cu"], s["ref"], need_grad=case["way"] == "step")
    out = dict(loss=r.loss, pair_loss=r.pair_loss, seq_logp=r.seq_logp, logp=r.logp)
    if case["way"] == "step":
        out["dlogits"] = tr.preference_backward(s["logits"], s["targets"], r)
    return out


# ---------------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_round_e4m3(v):
    """The nearest E4M3 value (ties to the even one) of 64-bit v, |v| <= 448: three bits after the leading one, spacing at least 2^-9."""
    spacing = torch.exp2(torch.clamp(torch.floor(torch.log2(v.abs().clamp(min=1e-300))), min=-6.0) - 3.0)
    return torch.round(v / spacing) * spacing


def _exact_codes(x):
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    full = torch.zeros((rows, nb * BLOCK), dtype=torch.float64, device=x.device)
    full[:, :cols] = x.double()
    full = full.view(rows, nb, BLOCK)
    amax = full.abs().max(2).values
    p = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -160) / 448.0))
    p = torch.where(amax > 448.0 * torch.exp2(p), p + 1, p)              # log2 may be off by a rounding at a power of two
    p = torch.where(amax <= 448.0 * torch.exp2(p - 1), p - 1, p).clamp(min=-127)
    return _exact_round_e4m3(full / torch.exp2(p)[:, :, None]).view(rows, -1)[:, :cols]


def _exact_value(codes, scales):
    codes = codes.view(torch.float8_e4m3fn).double()
    return codes * torch.exp2(scales.double() - 127.0)[:, torch.arange(codes.shape[1], device=codes.device) // BLOCK]


def _exact_norm(s, case):
    gate = s["gate"].double()[torch.arange(case["rows"], device="cuda") // _rows_per_gate(case)]
    w1, w2, c = s["post_gain"].double(), s["pre_gain"].double(), case["cols"]
    if case["way"] == "fwd":
        h, y = s["h"].double(), s["y"].double()
        ip = 1 / torch.sqrt(y.square().sum(1) / c + EPS)
        H = s["res_scale"] * h + gate * y * ip[:, None] * w1
        iq = 1 / torch.sqrt(H.square().sum(1) / c + EPS)
        out = dict(h_out=H, x=H * iq[:, None] * w2, inv_post=ip, inv_pre=iq)
        if case["saved"] == "codes":
            out |= dict(h_codes=_exact_codes(s["h"]), h_scales=None, y_codes=_exact_codes(s["y"]), y_scales=None)
        return out
    h, y = (_exact_value(*s[k]) if case["saved"] == "codes" else s[k].double() for k in ("h", "y"))
    ip, iq = s["inv_post"].double()[:, None], s["inv_pre"].double()[:, None]
    yh = y * ip
    xh = (s["res_scale"] * h + gate * yh * w1) * iq
    dx = s["dx"].double()
    d = s["dh_out"].double() + iq * (dx * w2 - xh * ((dx * w2 * xh).sum(1, keepdim=True) / c))
    dn = gate * d * w1
    dgate = torch.zeros((_gates(case), c), dtype=torch.float64, device="cuda")
    dgate.index_add_(0, torch.arange(case["rows"], device="cuda") // _rows_per_gate(case), d * yh * w1)
    return dict(dh=s["res_scale"] * d, dy=ip * (dn - yh * ((dn * yh).sum(1, keepdim=True) / c)), dpost_gain=(gate * d * yh).sum(0),
                dpre_gain=(dx * xh).sum(0), dgate=dgate)


def _exact_gate(s, case):
    if case["way"] == "fwd":
        g, u = s["g"].double(), s["u"].double()
        return dict(z=g * torch.sigmoid(g) * u, g_codes=_exact_codes(s["g"]), g_scales=None, u_codes=_exact_codes(s["u"]), u_scales=None)
    g, u, dz = _exact_value(*s["g"]), _exact_value(*s["u"]), s["dz"].double()
    sg = torch.sigmoid(g)
    return dict(dg=dz * u * (sg + g * sg * (1 - sg)), du=dz * g * sg)


def _exact_pref(s, case):
    rows, pairs, targets = case["rows"], case["pairs"], s["targets"]
    cu, ref = s["cu"].tolist(), s["ref"].double().tolist()
    lse = torch.cat([torch.logsumexp(s["logits"][i:i + 1024].double(), 1) for i in range(0, rows, 1024)])
    counted = (targets >= 0)
    at = torch.where(counted, targets, 0)
    logp = torch.where(counted, s["logits"].gather(1, at[:, None])[:, 0].double() - lse, 0.0)
    total = [float(logp[a:b].sum()) for a, b in zip(cu, cu[1:])]
    count = [max(1, int(counted[a:b].sum())) for a, b in zip(cu, cu[1:])]
    seq = [t / n if case["average"] else t for t, n in zip(total, count)]
    one = torch.ones((), dtype=torch.float64)
    losses, coef = [], torch.zeros(rows, dtype=torch.float64, device="cuda")
    for p in range(pairs):
        u = (seq[2 * p] - ref[2 * p]) - (seq[2 * p + 1] - ref[2 * p + 1])
        d = BETA * u * one
        if case["kind"] == "sigmoid":
            l = (1 - SMOOTHING) * torch.nn.functional.softplus(-d) + SMOOTHING * torch.nn.functional.softplus(d)
            du = float(BETA * (torch.sigmoid(d) - 1 + SMOOTHING))
        elif case["kind"] == "hinge":
            l, du = torch.relu(1 - d), -BETA if float(d) < 1 else 0.0
        else:
            l, du = (u - 1 / (2 * BETA)) ** 2 * one, 2 * (u - 1 / (2 * BETA))
        losses.append(float(l) - NLL_WEIGHT * total[2 * p] / count[2 * p])
        for j, sign in ((2 * p, 1.0), (2 * p + 1, -1.0)):
            c = sign * du / (count[j] if case["average"] else 1) - (NLL_WEIGHT / count[j] if sign > 0 else 0.0)
            coef[cu[j]:cu[j + 1]] = c / pairs
    out = dict(loss=torch.tensor(sum(losses) / pairs, dtype=torch.float64), pair_loss=torch.tensor(losses, dtype=torch.float64), seq_logp=torch.tensor(seq, dtype=torch.float64),
               logp=logp)
    if case["way"] == "step":
        coef = torch.where(counted, coef, 0.0)
        grad = torch.empty((rows, case["vocab"]), dtype=torch.float64, device="cuda")
        for i in range(0, rows, 1024):
            grad[i:i + 1024] = -coef[i:i + 1024, None] * torch.exp(s["logits"][i:i + 1024].double() - lse[i:i + 1024, None])
        grad[torch.arange(rows, device="cuda"), at] += coef
        out["dlogits"] = grad
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "gate": _exact_gate, "pref": _exact_pref}[case["op"]](s, case)
