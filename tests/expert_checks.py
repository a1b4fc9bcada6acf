"""Plain 64-bit implementations of the experts' operators and the error bounds their tests use, from the formulas of
include/zero_operators.h, on CPU tensors in the operators' types.

Bounds: products of 16-bit numbers are exact in fp32, of 32-bit ones off by U.  A sum of n products is off by at
most n units of the sum of their magnitudes; the matrix cores may cut where others round, so a unit is
2 U there.
"""
import torch

from operator_checks import U, normal, order, rng  # noqa: F401


def choice(tokens, k, experts, seed, none=0.0, only=None):
    """(index [tokens, k], offsets, order), int32: experts at random, `none` the share of slots without one, `only`
    the experts that are chosen at all."""
    g = rng(seed, tokens, k, experts)
    index = torch.randint(0, experts, (tokens, k), generator=g)
    if only is not None:
        index = torch.tensor(only)[index % len(only)]
    index[torch.rand(tokens, k, generator=g) < none] = -1
    offsets, placed = order(index, experts)
    return index.int(), torch.tensor(offsets, dtype=torch.int32), torch.tensor(placed, dtype=torch.int32)


def rows_of(mode, offsets, placed):
    """The rows of a matrix that lies as `mode` says, for the rows of the experts' order."""
    n = int(offsets[-1])
    slots = placed[:n].long()
    return torch.arange(n) if mode == 0 else slots // mode


def runs(offsets):
    ends = offsets.tolist()
    return [(e, a, b) for e, (a, b) in enumerate(zip(ends, ends[1:])) if a < b]


def product(x, w, offsets, placed, x_slots, y_slots, transposed, slots):
    """(y, its bound, which rows are written)."""
    xr, yr = rows_of(x_slots, offsets, placed), rows_of(y_slots, offsets, placed)
    x, w = x.double(), w.double()
    cols = w.shape[1] if transposed else w.shape[2]
    y, size = (torch.zeros(slots, cols, dtype=torch.float64) for _ in range(2))
    written = torch.zeros(slots, dtype=torch.bool)
    written[yr] = True
    for e, a, b in runs(offsets):
        m = w[e].t() if transposed else w[e]
        y[yr[a:b]] = x[xr[a:b]] @ m
        size[yr[a:b]] = x[xr[a:b]].abs() @ m.abs()
    return y, (x.shape[1] + 8) * 2 * U * size, written


def weight_backward(x, dy, offsets, placed, x_slots, dy_slots):
    """(dweight, its bound)."""
    xr, yr = rows_of(x_slots, offsets, placed), rows_of(dy_slots, offsets, placed)
    x, dy = x.double(), dy.double()
    experts = offsets.numel() - 1
    dw, bound = (torch.zeros(experts, x.shape[1], dy.shape[1], dtype=torch.float64) for _ in range(2))
    for e, a, b in runs(offsets):
        dw[e] = x[xr[a:b]].t() @ dy[yr[a:b]]
        bound[e] = (b - a + 8) * 2 * U * (x[xr[a:b]].abs().t() @ dy[yr[a:b]].abs())
    return dw, bound


def there(index, experts):
    return (index >= 0) & ((index < experts) if experts else True)


def mix(y, index, weight, base, experts=0):
    tokens, k = index.shape
    has = there(index, experts)[:, :, None]
    w = torch.ones(tokens, k) if weight is None else weight
    terms = torch.where(has, y.double().view(tokens, k, -1) * w.double()[:, :, None], 0.0)
    b = torch.zeros(tokens, y.shape[1], dtype=torch.float64) if base is None else base.double()
    return b + terms.sum(1), (k + 2) * U * (b.abs() + terms.abs().sum(1))


def mix_backward(dout, y, index, weight, experts=0):
    """(dy, dweight, its bound): a lane of 64 adds up its share in turn, then six steps."""
    tokens, k = index.shape
    has = there(index, experts)
    w = torch.ones(tokens, k) if weight is None else weight
    d = dout.double()
    dy = torch.where(has[:, :, None], w.double()[:, :, None] * d[:, None], 0.0).view(tokens * k, -1)
    terms = torch.where(has[:, :, None], y.double().view(tokens, k, -1) * d[:, None], 0.0)
    return dy, terms.sum(2), (dout.shape[1] / 64 + 16) * U * terms.abs().sum(2)
