"""Plain 64-bit implementations of zero_log_probs and its gradient and the error bounds their tests use, from the
formulas of include/zero_operators.h, on CPU tensors.

With x = (z - m) / temperature, fp32 holds x to 2 U |x| (the scale's rounding and its own), 2^x is off by 4 U beside
that, a thread adds up to max(64, vocab / 1024) terms in turn and 30 steps follow; the hardware's log2 is
off by 4 U of its value.
"""
import math

import torch

from operator_checks import NORMAL, U, normal, rng  # noqa: F401


def parts(z, tau):
    """(x, p, ln S, empty rows) in 64 bits."""
    z = z.double()
    m = z.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(1, keepdim=True)
    empty = (z == -math.inf).all(1)
    x = torch.where(z == -math.inf, -math.inf, (z - m) / tau)
    x[empty] = -math.inf
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    return x, torch.where(empty[:, None], 0.0, e / total), torch.log(total), empty


def mean(p, x, power=1):
    return torch.where(p > 0, p * torch.where(p > 0, x, 0.0).abs() ** power, torch.where(torch.isnan(p), p, 0.0)).sum(1)


def fp32(t):
    """-inf where a value is past fp32's range."""
    return torch.where(t < -(2.0 - 2.0 ** -24) * 2.0 ** 127, -math.inf, t)


def log_probs(z, tokens, k, tau):
    """A dict of (value, bound): logp, entropy; top_index; stats."""
    rows, vocab = z.shape
    x, p, log_sum, empty = parts(z, tau)
    adds = max(64, vocab / 1024) + 30
    first, second = mean(p, x), mean(p, x, 2)
    of_sum = (adds + 8 + 2 * first + 8 * log_sum[:, 0].abs()) * U       # ln S
    lp = fp32(torch.where(empty[:, None], -math.inf, x - log_sum))
    off = (of_sum[:, None] + 4 * U * x.abs()).nan_to_num(nan=0.0, posinf=0.0)
    out = {}
    if tokens is not None:
        at, has = tokens.long().clamp(0, vocab - 1)[:, None], (tokens >= 0) & (tokens < vocab)
        out["logp"] = torch.where(has, lp.gather(1, at)[:, 0], 0.0), off.gather(1, at)[:, 0]
    h = torch.where(empty, 0.0, log_sum[:, 0] + first)
    bound = of_sum + ((adds + 12) * first + 2 * second) * U + first * (adds + 8 + 2 * first) * U
    out["entropy"] = h, bound.nan_to_num(nan=0.0, posinf=0.0)
    if k:
        zz = z.float() + 0.0
        key = torch.where(torch.isnan(zz), -math.inf, zz)
        v, i = key.sort(dim=1, descending=True, stable=True)
        v, i = v[:, :k], i[:, :k]
        pad = k - v.shape[1]
        listed = v > -math.inf
        top = torch.where(listed, i, -1)
        tlp = torch.where(listed, lp.gather(1, i), -math.inf)
        tb = off.gather(1, i)
        out["top_index"] = torch.nn.functional.pad(top, (0, pad), value=-1)
        out["top_logp"] = (torch.nn.functional.pad(tlp, (0, pad), value=-math.inf), torch.nn.functional.pad(tb, (0, pad)))
    m = z.double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).amax(1)
    total = torch.where(empty, 0.0, torch.exp(log_sum[:, 0]))
    out["stats"] = (torch.stack([m, total, h], 1),
                    torch.stack([torch.zeros(rows, dtype=torch.float64), (of_sum * total).nan_to_num(nan=0.0, posinf=0.0),
                                 out["entropy"][1]], 1))
    return out


def backward(z, tokens, dlogp, dentropy, tau, scale):
    """(dlogits, its bound) for statistics rounded to fp32."""
    rows, vocab = z.shape
    x, p, log_sum, empty = parts(z, tau)
    lp = x - log_sum
    h = log_sum + mean(p, x)[:, None]
    g, size = torch.zeros_like(x), torch.zeros_like(x)
    xs = torch.where(p > 0, x.abs(), 0.0)
    off = (4 * xs + 40) * U
    if dlogp is not None:
        has = ((tokens >= 0) & (tokens < vocab))[:, None]
        at = tokens.long().clamp(0, vocab - 1)[:, None]
        up = torch.where(has, dlogp.double()[:, None], 0.0)
        g = (-up * p).scatter_add(1, at, up)
        size = up.abs() * p
        size = size.scatter_add(1, at, up.abs() / 10)  # 4 U of it
    if dentropy is not None:
        d = dentropy.double()[:, None]
        g = g - d * torch.where(p > 0, p * (lp + h), torch.where(torch.isnan(p), p, 0.0))
        size = size + d.abs() * p * (xs + log_sum.abs() + h)
    g = torch.where(empty[:, None], 0.0, g * scale / tau)
    bound = (size * off + NORMAL * 300) * abs(scale) / tau
    return g, torch.where(empty[:, None], 0.0, bound).nan_to_num(nan=0.0, posinf=0.0)
