"""Plain 64-bit forms of the operators of include/falqon_train.h, on the CPU, with the magnitudes that error bounds are derived from."""
import numpy as np
import torch

BF16_HALF_STEP = 2.0 ** -8      # relative: bf16 keeps 8 significant bits, so 1 + 2^-8 lies half-way between two values


def type_rounding(dtype):
    return BF16_HALF_STEP if dtype == torch.bfloat16 else 2.0 ** -24


def d(t):
    return None if t is None else t.detach().cpu().double()


def e4m3_values():
    """The 256 values of E4M3 (NaN for 0x7F and 0xFF), from the format's definition: 4 exponent bits, bias 7, 3 mantissa bits."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = np.nan if (c & 127) == 127 else -v if c & 128 else v
    return out


def encode(x):
    """Scale bytes [rows, blocks] and the values of the codes [rows, cols] of a checkpoint of x (float64 numpy), by definition: the
    smallest e >= 0 with amax * 2^(127 - e) <= 448, then the nearest E4M3 value, ties to the even code."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    grid = e4m3_values()[:127]                                   # 0 .. 448, ascending
    scales, vals = np.zeros((rows, nb), np.int64), np.empty((rows, cols))
    for b in range(nb):
        blk = x[:, 32 * b:32 * b + 32]
        amax = np.abs(blk).max(1)
        bad = ~np.isfinite(amax)
        e = np.zeros(rows, np.int64)
        safe = np.where(bad, 0.0, amax)
        for _ in range(255):
            e = np.where(safe * 2.0 ** (127.0 - e) > 448.0, e + 1, e)
        s = np.abs(np.where(bad[:, None], 0.0, blk)) * 2.0 ** (127.0 - e)[:, None]
        hi = np.clip(np.searchsorted(grid, s), 0, 126)           # grid[hi] >= s
        lo = np.maximum(hi - 1, 0)
        up, down = grid[hi] - s, s - grid[lo]
        code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
        v = np.copysign(grid[code], np.where(bad[:, None], 1.0, blk))
        vals[:, 32 * b:32 * b + 32] = np.where(bad[:, None], np.nan, v)
        scales[:, b] = np.where(bad, 255, e)
    return scales, vals


def decode(codes, scales):
    v = e4m3_values()[codes]
    e = scales.astype(np.int64)
    f = np.where(e == 255, np.nan, 2.0 ** (e - 127.0))
    return v * np.repeat(f, 32, axis=1)[:, :v.shape[1]]


class Norm:
    """The block norm in 64 bits; h, y, gains, gate as double tensors (gains and gate None: 1)."""

    def __init__(self, rows, cols, post=True, pre=True, post_gain=None, pre_gain=None, gate=None, rows_per_gate=None, res_scale=1.0,
                 gain_offset=0.0, eps=1e-6):
        self.rows, self.cols, self.post, self.pre, self.s, self.eps = rows, cols, post, pre, res_scale, eps
        one = torch.ones(cols, dtype=torch.float64)
        self.w1 = one if post_gain is None else gain_offset + post_gain
        self.w2 = one if pre_gain is None else gain_offset + pre_gain
        rpg = rows if rows_per_gate is None else rows_per_gate
        self.group = torch.arange(rows) // rpg
        self.gate = torch.ones((rows, cols), dtype=torch.float64) if gate is None else gate.view(-1, cols)[self.group]

    def forward(self, h, y):
        self.ip = 1 / torch.sqrt((y * y).mean(1, keepdim=True) + self.eps) if self.post else torch.ones((self.rows, 1), dtype=torch.float64)
        n = y * self.ip * (self.w1 if self.post else 1.0)
        H = self.gate * n + (0 if h is None else self.s * h)
        self.H_size = (self.gate * n).abs() + (0 if h is None else (self.s * h).abs())
        self.iq = 1 / torch.sqrt((H * H).mean(1, keepdim=True) + self.eps)
        return H, H * self.iq * self.w2

    def backward(self, dx, dh_out, h, y, ip, iq):
        """Gradients and, for each, the sum of the magnitudes that were added up (error bounds are multiples of it)."""
        w1 = self.w1 if self.post else torch.ones(self.cols, dtype=torch.float64)
        ip = ip[:, None] if self.post else torch.ones((self.rows, 1), dtype=torch.float64)
        yh = y * ip
        H = self.gate * yh * w1 + (0 if h is None else self.s * h)
        Hs = (self.gate * yh * w1).abs() + (0 if h is None else (self.s * h).abs())
        g = torch.zeros_like(y) if dh_out is None else dh_out
        if self.pre:
            iq = iq[:, None]
            xh, xs, a = H * iq, Hs * iq, dx * self.w2
            dd = g + iq * (a - xh * (a * xh).mean(1, keepdim=True))
            ds = g.abs() + iq * (a.abs() + xs * (a.abs() * xs).mean(1, keepdim=True))
        else:
            xh = xs = torch.zeros_like(y)
            dx = torch.zeros_like(y)
            dd, ds = g, g.abs()
        b, bs = self.gate * dd * w1, (self.gate * w1).abs() * ds
        if self.post:
            dy = ip * (b - yh * (b * yh).mean(1, keepdim=True))
            dys = ip * (bs + yh.abs() * (bs * yh.abs()).mean(1, keepdim=True))
        else:
            dy, dys = b, bs
        groups = int(self.group.max()) + 1
        sums = lambda t: torch.zeros((groups, self.cols), dtype=torch.float64).index_add_(0, self.group, t)  # noqa: E731
        return dict(dh=(self.s * dd, abs(self.s) * ds), dy=(dy, dys), dpost_gain=((self.gate * dd * yh).sum(0), (self.gate.abs() * ds * yh.abs()).sum(0)),
                    dpre_gain=((dx * xh).sum(0), (dx.abs() * xs).sum(0)), dgate=(sums(dd * yh * w1), sums(ds * (yh * w1).abs())))


def sequence_logprob(logits, targets, cu, average):
    logits, targets = d(logits), targets.cpu()
    rows, vocab = logits.shape
    counted = (targets >= 0) & (targets < vocab)
    inside = torch.zeros(rows, dtype=torch.bool)
    logp = torch.zeros(rows, dtype=torch.float64)
    for r in range(rows):
        if counted[r]:
            logp[r] = torch.log_softmax(logits[r], 0)[targets[r]]       # differences from the maximum first: a row of lowest values is uniform
    seq, count = [], []
    for a, b in zip(cu, cu[1:]):
        inside[a:b] = True
        n = int(counted[a:b].sum())
        t = logp[a:b].sum()
        seq.append(t / max(n, 1) if average else t)
        count.append(n)
    return torch.stack(seq), torch.where(inside, logp, 0.0), count, counted & inside


def preference(logits, targets, cu, ref, kind, beta, margin, smoothing, average, nll_weight):
    """loss, pair_loss, seq_logp, logp, dlogits in 64 bits; differentiable where logits is a double tensor that requires it."""
    seq, logp, count, counted = sequence_logprob(logits, targets, cu, average)
    ref = torch.zeros_like(seq) if ref is None else d(ref)
    u = (seq - ref)[0::2] - (seq - ref)[1::2]
    D = beta * u - margin
    if kind == "sigmoid":
        sp = torch.nn.functional.softplus
        l = (1 - smoothing) * sp(-D) + smoothing * sp(D)
        du = beta * (torch.sigmoid(D) - 1 + smoothing)
    elif kind == "hinge":
        l, du = torch.relu(1 - D), torch.where(D < 1, -beta, 0.0).double()
    else:
        l, du = (u - margin - 1 / (2 * beta)) ** 2, 2 * (u - margin - 1 / (2 * beta))
    pairs = len(u)
    coef = torch.zeros(len(logp), dtype=torch.float64)
    total = [logp[a:b].sum() for a, b in zip(cu, cu[1:])]
    pair_loss = []
    for p in range(pairs):
        nll = nll_weight / max(count[2 * p], 1)
        pair_loss.append(l[p] - nll * total[2 * p] if nll else l[p])
        for j, sign in ((2 * p, 1.0), (2 * p + 1, -1.0)):
            c = sign * du[p] / (max(count[j], 1) if average else 1) - (nll if sign > 0 else 0.0)
            coef[cu[j]:cu[j + 1]] = c / pairs
    coef = torch.where(counted, coef, 0.0)
    x, t = d(logits), targets.cpu()
    p = torch.where(counted[:, None], torch.softmax(x, 1), 0.0)
    one = torch.zeros_like(p)
    one[counted, t[counted]] = 1.0
    pair_loss = torch.stack(pair_loss)
    return dict(loss=pair_loss.mean(), pair_loss=pair_loss, seq_logp=seq, logp=logp, dlogits=coef[:, None] * (one - p), size=coef.abs()[:, None] * (one + p),
                u=u, counted=counted, onehot=one, p=p)
