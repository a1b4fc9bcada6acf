"""Plain 64-bit implementations of the training operators and the error bounds their tests use.

Every function takes CPU tensors in the operators' types and computes in float64 from the formulas of
include/zero_operators.h.  Bounds: U is fp32's unit roundoff and UNIT a type's; TINY is half
the type's least spacing, what a rounding into its subnormal range can add.  The constants count
the fp32 operations on the longest path to a value (a lane's own sum, then at most 16 steps
across lanes and waves), with the hardware's 2^x and log2 taken as 2 units each.
"""
import math

import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = (torch.float16, torch.bfloat16, torch.float32)
NORMAL = 2.0 ** -126   # below it the hardware's 2^x is 0


def rng(*seed):
    return torch.Generator().manual_seed(sum(int(s) * 1009 ** i for i, s in enumerate(seed)) % (1 << 31))


def normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, dtype=torch.float64) * std


def within(got, want, bound, what):
    """got (any type) against float64 want: NaN and inf where want has them, else |got - want| <= bound."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    plain = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaN elsewhere" % what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), "%s: inf elsewhere" % what
    err = (got - want).abs()[plain]
    lim = bound.expand_as(want)[plain] if torch.is_tensor(bound) else torch.full_like(err, bound)
    bad = ~(err <= lim)
    if bad.any():
        i = int((err - lim).argmax())
        raise AssertionError("%s: %d of %d off, worst |%g - %g| = %g > %g" % (
            what, int(bad.sum()), err.numel(), got[plain][i], want[plain][i], err[i], lim[i]))


# --- norm -----------------------------------------------------------------------

#: a lane sums up to 64 squares, then 6 steps in its wave and 15 across waves; half of it in the root
ROOT = 48 * U


def rms_norm(h, w, eps):
    """(rstd, y) of the rounded sum h."""
    h, w = h.double(), w.double()
    rstd = (h.square().mean(1) + eps).rsqrt()
    return rstd, h * rstd[:, None] * w


def scales(y, group):
    cols = y.shape[1]
    parts = y.split(group or cols, dim=1)
    amax = torch.stack([p.abs().amax(1) for p in parts], 1)
    return amax.clamp(min=2.0 ** -100) / 448.0


def spread(scale, cols, group):
    return scale.repeat_interleave(group or cols, 1)[:, :cols]


def check_e4m3(codes, y, group, what):
    """Each code is what y / scale rounds to, on one side or the other of a relative 1e-5 (ROOT and a few
    operations more are 4e-6)."""
    v = y / spread(scales(y, group), y.shape[1], group)
    lo, hi = ((v * (1 + s)).clamp(-448, 448).float().to(torch.float8_e4m3fn).float() for s in (-1e-5, 1e-5))
    got = codes.detach().cpu().view(torch.float8_e4m3fn).float()
    bad = (got != lo) & (got != hi)
    assert not bad.any(), "%s: %d codes, e.g. %g of %g" % (what, int(bad.sum()), got[bad][0], v[bad][0])


def rms_norm_backward(dy, h, w, rstd, dh):
    """(dx, dw) and the bounds of their fp32 errors."""
    dy, h, w, rstd = dy.double(), h.double(), w.double(), rstd.double()[:, None]
    n, g = h * rstd, dy * w
    mean, size = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    dx = rstd * (g - n * mean)
    bound = rstd * (4 * U * g.abs() + n.abs() * (6 * U * mean.abs() + 2 * ROOT * size))
    if dh is not None:
        dx = dx + dh.double()
        bound = bound + U * dx.abs()
    each = dy * n
    # a workgroup's rows in turn (rows / 512, at most 64 of them in these tests), its segments, then the partial sums
    return dx, each.sum(0), bound, 160 * U * each.abs().sum(0)


# --- routing ----------------------------------------------------------------------

def route(logits, bias, score, groups, top_groups, group_top, k, renormalise, scale):
    """(index, weight, key): keys of softmax are fp32 sums, as defined; of sigmoid in float64."""
    z = logits.double()
    rows, experts = z.shape
    b = torch.zeros(experts) if bias is None else bias
    out = (z == -math.inf) | (b == -math.inf)
    if score == "softmax":
        key = (logits.float() + b).double()
    else:
        key = torch.sigmoid(z) + b.double()
    key = key.masked_fill(out | torch.isnan(key), -math.inf)
    left = key
    if groups > 1:
        best = key.view(rows, groups, -1).topk(group_top, dim=2).values
        s = best.sum(2)
        if score == "softmax" and group_top == 2:
            s = (best[:, :, 0].float() + best[:, :, 1].float()).double()
        s = s.masked_fill(torch.isnan(s), -math.inf)
        place = s.argsort(dim=1, descending=True, stable=True).argsort(dim=1)
        stays = (place < top_groups) & (s > -math.inf)
        left = key.masked_fill(~stays.repeat_interleave(experts // groups, 1), -math.inf)
    v, i = left.sort(dim=1, descending=True, stable=True)
    index = torch.where(v[:, :k] > -math.inf, i[:, :k], -1)
    return index, weights(z, out, index, score, renormalise, scale), left


def weights(z, out, index, score, renormalise, scale):
    none, at = index < 0, index.clamp(min=0)
    z = z.masked_fill(out, -math.inf)
    if score == "softmax":
        over = z.gather(1, at).masked_fill(none, -math.inf) if renormalise else z
        top = over.nan_to_num(nan=-math.inf, neginf=-math.inf, posinf=math.inf).amax(1, keepdim=True)
        w = (z.gather(1, at) - top).exp() / (over - top).exp().sum(1, keepdim=True)
    else:
        w = torch.sigmoid(z.gather(1, at)).masked_fill(none, 0.0)
        if renormalise:
            w = w / w.sum(1, keepdim=True).clamp(min=2.0 ** -126)
    w = torch.where(torch.isnan(z).any(1, keepdim=True), math.nan, w * scale)
    return w.masked_fill(none, 0.0)


def route_backward(logits, bias, index, dweight, score, renormalise, scale):
    """dlogits by the written-out derivative, and the sum of the magnitudes that it is made of."""
    z = logits.double()
    b = torch.zeros(z.shape[1]) if bias is None else bias
    out = (z == -math.inf) | (b == -math.inf)
    none, at = index < 0, index.clamp(min=0).long()
    d = (dweight.double() * scale).masked_fill(none, 0.0)
    if score == "softmax":
        zz = z.masked_fill(out, -math.inf)
        over = zz.gather(1, at).masked_fill(none, -math.inf) if renormalise else zz
        top = over.amax(1, keepdim=True)
        total = (over - top).exp().sum(1, keepdim=True)
        p = ((zz.gather(1, at) - top).exp() / total).masked_fill(none, 0.0)
        mean, size = (p * d).sum(1, keepdim=True), (p * d).abs().sum(1, keepdim=True)
        if renormalise:
            g = torch.zeros_like(z).scatter_add(1, at, p * (d - mean))
            m = torch.zeros_like(z).scatter_add(1, at, p * (d.abs() + size))
        else:
            s = ((zz - top).exp() / total).masked_fill(out, 0.0)
            g = (-s * mean).scatter_add(1, at, p * d)
            m = (s * size).scatter_add(1, at, (p * d).abs())
    else:
        s = torch.sigmoid(z.gather(1, at)).masked_fill(none, 0.0)
        t, size = d, d.abs()
        if renormalise:
            total = s.sum(1, keepdim=True).clamp(min=2.0 ** -126)
            t = (d - (d * s).sum(1, keepdim=True) / total) / total
            size = (d.abs() + (d * s).abs().sum(1, keepdim=True) / total) / total
        # 1 - s loses what s lacks of 1: U of s, not of the difference
        g = torch.zeros_like(z).scatter_add(1, at, t * s * (1 - s))
        m = torch.zeros_like(z).scatter_add(1, at, size * s)
    return g, m


def order(index, experts):
    flat = index.reshape(-1).tolist()
    runs = [[] for _ in range(experts)]
    for s, e in enumerate(flat):
        if 0 <= e < experts:
            runs[e].append(s)
    offsets = [0]
    for r in runs:
        offsets.append(offsets[-1] + len(r))
    got = [s for r in runs for s in r]
    return offsets, got + [-1] * (len(flat) - len(got))


# --- distillation -------------------------------------------------------------------

def distill(z, index, teacher, labels, soft, hard, tau, weight, scale, dloss=None):
    """(loss, its bound, dlogits, its bound) in float64; the bounds are of fp32's errors."""
    z = z.double()
    rows, vocab = z.shape
    weight = torch.ones(rows, dtype=torch.float64) if weight is None else weight.double()
    up = weight * scale * (1.0 if dloss is None else dloss.double())
    m = z.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(1, keepdim=True)
    loss = torch.zeros(rows, dtype=torch.float64)
    off = torch.zeros(rows, dtype=torch.float64)
    g, gb = torch.zeros_like(z), torch.zeros_like(z)

    def log_soft(t):  # log q and the units by which q may be off
        x = (z - m) / t
        lq = x - torch.log(torch.exp(x).sum(1, keepdim=True))
        return lq, (4 * x.abs().masked_fill(x == -math.inf, 0.0) + 60) * U

    if index is not None and index.shape[1] and soft:
        absent = (index < 0) | (index >= vocab) | (teacher.double() == -math.inf)
        at = index.long().clamp(0, vocab - 1)
        has = (~absent).any(1, keepdim=True)
        t = (teacher.double() / tau).masked_fill(absent, -math.inf)
        t = t - t.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(1, keepdim=True)
        p = torch.where(absent, 0.0, torch.exp(t))
        total = p.sum(1, keepdim=True)
        p = torch.where(has, p / total, 0.0)
        lp = t - torch.log(total)
        lq, units = log_soft(tau)
        lqa = lq.gather(1, at)
        zero = absent | (p < NORMAL)
        each = torch.where(zero, 0.0, p * (lp - lqa))
        punits = (4 * torch.where(zero, 0.0, t.abs()) + 60) * U
        loss = loss + soft * tau ** 2 * torch.where(has[:, 0], each.sum(1), 0.0)
        # an entry's share and its two logarithms, then the sum of up to 16 entries a thread and the steps across
        size = torch.where(zero, 0.0, p * (lp.abs() + lqa.abs() + 1))
        off = off + abs(soft) * tau ** 2 * (size * (punits + units.gather(1, at) + 40 * U)).sum(1)
        q = torch.where(has, lq.exp(), 0.0)
        g = g + soft * tau * torch.where(has, lq.exp(), 0.0)
        gb = gb + abs(soft) * tau * (q * units + torch.where(has, NORMAL, 0.0))
        g = g.scatter_add(1, at, -soft * tau * p)
        gb = gb.scatter_add(1, at, abs(soft) * tau * (p * punits + NORMAL))
    if labels is not None and hard:
        has = ((labels >= 0) & (labels < vocab))[:, None]
        at = labels.long().clamp(0, vocab - 1)[:, None]
        lq, units = log_soft(1.0)
        l = lq.gather(1, at)
        loss = loss + torch.where(has, -hard * l, 0.0)[:, 0]
        off = off + torch.where(has, abs(hard) * (l.abs() + 1) * (units.gather(1, at) + 8 * U), 0.0)[:, 0]
        g = g + torch.where(has, hard * lq.exp(), 0.0)
        gb = gb + torch.where(has, abs(hard) * (lq.exp() * units + NORMAL), 0.0)
        g = g.scatter_add(1, at, has.double() * -hard)
        gb = gb.scatter_add(1, at, has.double() * (abs(hard) * 4 * U))
    seen = weight != 0
    loss = torch.where(seen, weight * loss, 0.0)
    off = torch.where(seen, weight.abs() * off, 0.0) + 2 * U * loss.abs()
    g = torch.where(seen[:, None], up[:, None] * g, 0.0)
    gb = torch.where(seen[:, None], up[:, None].abs() * gb, 0.0) + 6 * U * g.abs()
    return loss, off, g, gb


def rounded(bound, want, dtype):
    """A bound of the fp32 value with the rounding into `dtype` added; what overflows is inf on both sides."""
    return bound * (1 + UNIT[dtype]) + UNIT[dtype] * want.abs() + TINY[dtype]
