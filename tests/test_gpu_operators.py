"""The training operators on the GPU against plain 64-bit implementations (operator_checks.py), at the sizes,
strides and masks where they can go wrong; gradients also against differences of the forward.  Outputs lie between
guard elements, which must stay."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_checks as C  # noqa: E402

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
GUARD = 37  # elements on both sides of an output's buffer


@pytest.fixture(scope="module")
def zo():
    from paper_1910_02054_amd import operators
    assert torch.cuda.is_available()
    return operators


class Out:
    """An output matrix on the device, rows `pad` elements further apart than its columns and the first `lead`
    elements past an aligned address; everything around it holds a byte pattern that must stay."""

    def __init__(self, rows, cols, dtype, pad=0, lead=0):
        size = torch.empty(0, dtype=dtype).element_size()
        n = GUARD * 2 + lead + rows * (cols + pad)
        self.raw = torch.full((n * size,), 0xA5, dtype=torch.uint8, device="cuda")
        flat = self.raw.view(dtype)
        self.view = flat[GUARD + lead:GUARD + lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        self.mask = torch.ones(n, dtype=torch.bool, device="cuda")
        self.mask[GUARD + lead:GUARD + lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = False
        self.size = size

    def guards_intact(self):
        return bool((self.raw.view(-1, self.size)[self.mask] == 0xA5).all())


def put(t, pad=0, lead=0):
    """A matrix on the device with its rows `pad` elements further apart; the elements between them are NaN."""
    o = Out(t.shape[0], t.shape[1], t.dtype, pad, lead)
    o.raw.view(t.dtype).fill_(math.nan)
    o.view.copy_(t)
    return o.view


# --- norm -----------------------------------------------------------------------

SIZES = [(1, 1), (3, 5), (40, 64), (5, 127), (33, 128), (7, 129), (9, 512), (6, 513), (5, 1024), (3, 1603), (4, 2048),
         (3, 2049), (2, 4096), (3, 4097), (2, 8192), (3, 8200), (2, 16384), (1, 25600), (2, 32767), (1, 32768)]


def norm_inputs(rows, cols, dtype, seed):
    g = C.rng(seed, rows, cols)
    big = torch.where(torch.rand(cols, generator=g) < 0.02, 20.0, 1.0)
    return (C.normal(g, rows, cols, std=0.5).to(dtype), (C.normal(g, rows, cols) * big).to(dtype),
            (1 + 0.1 * C.normal(g, cols)).to(dtype))


def check_norm(zo, rows, cols, dtype, group=0, residual=True, pad=0, lead=0, in_place=False, x=None, r=None,
               eps=1e-6, seed=1):
    xs, rs, w = norm_inputs(rows, cols, dtype, seed)
    x, r = xs if x is None else x, rs if r is None else r
    h = (x.float() + r.float()).to(dtype) if residual else x
    rstd, y = C.rms_norm(h, w, eps)
    ng = -(-cols // group) if group else 1
    oh, oy, oq = Out(rows, cols, dtype, pad, lead), Out(rows, cols, dtype, pad, lead), Out(rows, cols, torch.uint8, pad)
    os_, orr = Out(rows, ng, F32), Out(rows, 1, F32)
    dx, dr = put(x, pad, lead), put(r, pad, lead) if residual else None
    if in_place:
        oh.view.copy_(r)
        oy.view.copy_(x)
        dx, dr = oy.view, oh.view
    zo.zero_rms_norm(dx, w.cuda(), eps, residual=dr, h=oh.view if residual else None, y=oy.view, q8=oq.view,
                     scale=os_.view, group=group, rstd=orr.view)
    torch.cuda.synchronize()
    for o in (oh, oy, oq, os_, orr):
        assert o.guards_intact()
    if residual:
        assert torch.equal(oh.view.cpu(), h)
    C.within(orr.view[:, 0], rstd, (C.ROOT + 4 * C.U) * rstd, "rstd")
    C.within(oy.view, y, C.rounded((C.ROOT + 8 * C.U) * y.abs(), y, dtype), "y")
    s = C.scales(y, group)
    C.within(os_.view, s, (C.ROOT + 10 * C.U) * s, "scale")
    if torch.isfinite(y).all():
        C.check_e4m3(oq.view.contiguous(), y, group, "q8")
    return oh, oy, oq, os_, orr


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_norm_sizes(zo, rows, cols, dtype):
    for group in (0, 128):
        check_norm(zo, rows, cols, dtype, group, residual=(rows + cols) % 2 == 0)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("group", (0, 32, 64, 128, 256))
@pytest.mark.parametrize("cols", (31, 100, 256, 257, 640, 2080))
def test_norm_groups(zo, group, cols, dtype):
    check_norm(zo, 9, cols, dtype, group)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("pad,lead", ((0, 1), (3, 0), (8, 3), (64, 0)))
def test_norm_strides_and_in_place(zo, pad, lead, dtype):
    for cols in (65, 1600, 4100):
        check_norm(zo, 5, cols, dtype, 64, pad=pad, lead=lead)
        check_norm(zo, 5, cols, dtype, 0, pad=pad, lead=lead, in_place=True)


@pytest.mark.parametrize("dtype", C.TYPES)
def test_norm_special_rows(zo, dtype):
    cols = 300
    x, r, _ = norm_inputs(6, cols, dtype, 3)
    x[0], r[0] = 0.0, 0.0           # nothing but eps under the root, nothing to scale
    x[1, 7] = math.nan              # the whole row is NaN
    x[2, 200] = math.inf            # rstd 0, and NaN where 0 meets the infinity
    x[3], r[3] = 1e-30, 0.0         # squares below fp32's range (in fp16 they are 0 already)
    x[4], r[4] = torch.finfo(dtype).max, 0.0
    r[5] = -x[5]                    # the sum cancels
    if dtype != F16:                # squares of the largest values leave fp32's range, as a mean of fp32 does
        x[4] = 1e15
    xs = x.double() + r.double()
    assert torch.isfinite(xs[4]).all()
    h = (x.float() + r.float()).to(dtype)
    oh, oy, oq, os_, orr = check_rows(zo, x, r, h, cols, dtype)
    assert torch.isnan(oy.view[1]).all() and torch.isnan(os_.view[1]).all() and torch.isnan(orr.view[1]).all()
    assert (oq.view[1].cpu() & 0x7F == 0x7F).all()
    assert orr.view[2, 0] == 0 and torch.isnan(oy.view[2, 200]) and (oy.view[2, :200] == 0).all()
    assert (oq.view[0] == 0).all() and os_.view[0, 0].item() == pytest.approx(2.0 ** -100 / 448, rel=1e-6)


def check_rows(zo, x, r, h, cols, dtype):
    rows = x.shape[0]
    w = norm_inputs(rows, cols, dtype, 3)[2]
    oh, oy, oq = Out(rows, cols, dtype), Out(rows, cols, dtype), Out(rows, cols, torch.uint8)
    ng = -(-cols // 128)
    os_, orr = Out(rows, ng, F32), Out(rows, 1, F32)
    zo.zero_rms_norm(put(x), w.cuda(), 1e-6, residual=put(r), h=oh.view, y=oy.view, q8=oq.view, scale=os_.view,
                     group=128, rstd=orr.view)
    torch.cuda.synchronize()
    rstd, y = C.rms_norm(h, w, 1e-6)
    ok = [i for i in range(rows) if i not in (1, 2)]
    C.within(orr.view[ok, 0], rstd[ok], (C.ROOT + 4 * C.U) * rstd[ok], "rstd")
    C.within(oy.view[ok], y[ok], C.rounded((C.ROOT + 8 * C.U) * y[ok].abs(), y[ok], dtype), "y")
    C.check_e4m3(oq.view[ok].contiguous(), y[ok], 128, "q8")
    return oh, oy, oq, os_, orr


def test_norm_partial_outputs_and_no_rows(zo):
    x, r, w = (t.cuda() for t in norm_inputs(4, 100, F16, 5))
    y, h = torch.empty_like(x), torch.empty_like(x)
    zo.zero_rms_norm(x, w, 1e-6, residual=r, h=h, y=y)
    only = torch.empty_like(x)
    zo.zero_rms_norm(x, w, 1e-6, residual=r, y=only)      # the sum is not wanted
    assert torch.equal(only, y)
    zo.zero_rms_norm(h, w, 1e-6, y=only)                  # the sum as input: the same rows
    assert torch.equal(only, y)
    wide = torch.empty(4, 200, dtype=F16, device="cuda")  # columns of one buffer
    wide[:, :100] = x
    zo.zero_rms_norm(wide[:, :100], w, 1e-6, residual=r, y=wide[:, 100:])
    assert torch.equal(wide[:, 100:], y) and torch.equal(wide[:, :100], x)
    none = torch.empty(0, 100, dtype=F16, device="cuda")
    zo.zero_rms_norm(none, w, 1e-6, y=torch.empty_like(none))
    three = torch.empty(2, 2, 100, dtype=F16, device="cuda")
    zo.zero_rms_norm(x.view(2, 2, 100), w, 1e-6, residual=r, y=three)
    assert torch.equal(three.view(4, 100), y)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,cols", ((1, 1), (1, 8192), (2, 127), (17, 64), (100, 128), (5, 513), (1030, 200),
                                       (2055, 24), (37, 1603), (520, 2048), (515, 2049), (9, 4100), (3, 8200),
                                       (2, 25600), (2, 32768)))
def test_norm_backward(zo, rows, cols, dtype):
    for residual, pad in ((True, 0), (False, 5)):
        g = C.rng(7, rows, cols)
        h, dy, dh = (C.normal(g, rows, cols).to(dtype) for _ in range(3))
        w = (1 + 0.1 * C.normal(g, cols)).to(dtype)
        rstd = C.rms_norm(h, w, 1e-6)[0].float()
        dx, dw, bx, bw = C.rms_norm_backward(dy, h, w, rstd, dh if residual else None)
        ox, ow = Out(rows, cols, dtype, pad), Out(1, cols, dtype)
        n = zo.zero_rms_norm_workspace(rows, cols)
        assert n <= 1024 * cols
        room = Out(1, n, F32)
        args = (put(dy, pad), put(h, pad), w.cuda(), rstd.cuda())
        kw = dict(dh=put(dh, pad) if residual else None)
        zo.zero_rms_norm_backward(*args, ox.view, ow.view[0], room.view[0], **kw)
        torch.cuda.synchronize()
        assert ox.guards_intact() and ow.guards_intact() and room.guards_intact()
        C.within(ox.view, dx, C.rounded(bx, dx, dtype), "dx")
        C.within(ow.view[0], dw, C.rounded(bw, dw, dtype), "dw")
        # the same bits again, and in place
        again = torch.empty(cols, dtype=dtype, device="cuda")
        mine = args[0].clone()
        zo.zero_rms_norm_backward(mine, *args[1:], mine, again, room.view[0], **kw)
        assert torch.equal(again, ow.view[0]) and torch.equal(mine, ox.view)


def test_norm_backward_without_rows_and_with_a_bad_one(zo):
    none, w = torch.empty(0, 50, dtype=F16, device="cuda"), torch.ones(50, dtype=F16, device="cuda")
    dw = torch.full((50,), 7.0, dtype=F16, device="cuda")
    zo.zero_rms_norm_backward(none, none.clone(), w, torch.empty(0, device="cuda"), none.clone(), dw)
    assert (dw == 0).all()
    g = C.rng(11)
    h, dy = (C.normal(g, 4, 50).to(F16).cuda() for _ in range(2))
    dy[2, 3] = math.inf  # an overflowed gradient reaches dx's row and dw's column, and stays out of other rows
    rstd = C.rms_norm(h.cpu(), w.cpu(), 1e-6)[0].float().cuda()
    dx = torch.empty_like(h)
    zo.zero_rms_norm_backward(dy, h, w, rstd, dx, dw, torch.empty(4 * 50, device="cuda"))
    assert not torch.isfinite(dx[2]).any() and torch.isfinite(dx[[0, 1, 3]]).all()
    assert not math.isfinite(dw[3].item()) and torch.isfinite(dw[:3]).all() and torch.isfinite(dw[4:]).all()


def test_norm_gradient_against_differences(zo):
    """d sum(y dy) / dx by central differences of the fp32 forward: step 2^-6, whose curvature term and rounding
    (2^-24 * 40 terms / 2^-6) stay under 2e-3."""
    g = C.rng(13)
    x, dy = (C.normal(g, 3, 40).float() for _ in range(2))
    w = (1 + 0.1 * C.normal(g, 40)).float()
    rstd = torch.empty(3, device="cuda")
    y = torch.empty(3, 40, device="cuda")
    zo.zero_rms_norm(x.cuda(), w.cuda(), 1e-6, y=y, rstd=rstd)
    dx, dw = torch.empty(3, 40, device="cuda"), torch.empty(40, device="cuda")
    zo.zero_rms_norm_backward(dy.cuda(), x.cuda(), w.cuda(), rstd, dx, dw, torch.empty(3 * 40, device="cuda"))
    step = 2.0 ** -6
    for r, c in ((0, 0), (1, 17), (2, 39)):
        both = []
        for s in (step, -step):
            xs = x.clone()
            xs[r, c] += s
            zo.zero_rms_norm(xs.cuda(), w.cuda(), 1e-6, y=y)
            both.append((y.cpu().double() * dy.double()).sum())
        assert abs(float((both[0] - both[1]) / (2 * step)) - dx[r, c].item()) < 2e-3


# --- routing ----------------------------------------------------------------------

ROUTES = [  # rows, experts, k, groups, top_groups, group_top
    (1, 1, 1, 1, 1, 1), (1, 8, 2, 1, 1, 1), (3, 7, 7, 1, 1, 1), (65, 64, 6, 1, 1, 1), (33, 60, 4, 4, 2, 2),
    (40, 256, 8, 8, 4, 2), (17, 384, 10, 1, 1, 1), (9, 1024, 16, 1, 1, 1), (5, 1024, 64, 64, 20, 1),
    (12, 1023, 5, 33, 7, 2), (21, 160, 6, 8, 3, 1), (300, 16, 1, 1, 1, 1), (50, 96, 33, 3, 2, 2), (8, 66, 10, 33, 3, 2)]


def route_inputs(rows, experts, dtype, seed, bias, grid=True):
    """Logits in steps of 1/4 (many ties; distinct scores lie far apart) and a bias in steps of 1/64."""
    g = C.rng(seed, rows, experts)
    z = C.normal(g, rows, experts, std=1.5)
    z = (z * 4).round() / 4 if grid else z
    b = torch.randint(-8, 9, (experts,), generator=g).float() / 64 if bias else None
    return z.to(dtype), b


def clear_cut(key):
    """Whether distinct keys of every row differ by more than fp32 can confuse."""
    v = key.sort(1).values
    gap = (v[:, 1:] - v[:, :-1])[torch.isfinite(v[:, :-1]) & torch.isfinite(v[:, 1:])]
    return bool(((gap < 1e-12) | (gap > 1e-6)).all())


def run_route(zo, z, b, k, pad=0, **kw):
    rows = z.shape[0]
    oi, ow = Out(rows, k, torch.int32), Out(rows, k, F32)
    zo.zero_route(put(z, pad), oi.view, ow.view, bias=None if b is None else b.cuda(), **kw)
    torch.cuda.synchronize()
    assert oi.guards_intact() and ow.guards_intact()
    return oi.view.cpu().long(), ow.view


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
@pytest.mark.parametrize("shape", ROUTES)
def test_route(zo, shape, score, dtype):
    rows, experts, k, groups, top, per = shape
    for renorm, bias, scale, pad in ((True, True, 2.5, 0), (False, False, 1.0, 3)):
        z, b = route_inputs(rows, experts, dtype, 17, bias)
        index, w, key = C.route(z, b, score, groups, top, per, k, renorm, scale)
        assert clear_cut(key)
        got, gw = run_route(zo, z, b, k, pad, score=score, groups=groups, top_groups=top, group_top=per,
                            renormalise=renorm, scale=scale)
        assert torch.equal(got, index)
        # exponents of up to 12 units of ln 2 scale, a sum of 1024 terms (16 a lane), a division, the scale
        C.within(gw, w, 120 * C.U * w.abs() + C.NORMAL, "weight")


@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
def test_route_any_logits(zo, score):
    """Keys a few units apart may fall either way: the chosen ones' keys do not rise, and none left is larger."""
    z, b = route_inputs(200, 128, F32, 19, True, grid=False)
    _, _, key = C.route(z, b, score, 8, 8, 2, 8, True, 1.0)
    got, gw = run_route(zo, z, b, 8, score=score, groups=8, top_groups=8, group_top=2)
    v = key.gather(1, got)
    assert (v[:, 1:] <= v[:, :-1] + 4 * C.U).all()
    rest = key.scatter(1, got, -math.inf).amax(1)
    assert (rest <= v[:, -1] + 4 * C.U).all()
    out = torch.zeros_like(z, dtype=torch.bool)
    w = C.weights(z.double(), out, got, score, True, 1.0)
    C.within(gw, w, 120 * C.U * w, "weight")


@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
@pytest.mark.parametrize("groups,per", ((1, 1), (4, 1), (4, 2)))
def test_route_masks(zo, score, groups, per):
    experts, k, inf = 32, 6, math.inf
    for renorm in (True, False):
        z, b = route_inputs(12, experts, F32, 23, True)
        z[0] = -inf                          # no expert at all
        z[1, 3:] = -inf                      # three are left
        z[2] = torch.finfo(F32).min          # all at the lowest value: a tie, by index
        z[3, ::2] = torch.finfo(F32).min
        z[4, 5] = math.nan                   # not chosen; the weights say so
        z[5] = math.nan
        z[6, 9] = inf
        z[7] = 0.0
        z[7, 1::2] = -0.0                    # equal to 0: by index
        b[4] = -inf                          # an expert that is out
        z[8, 4] = math.nan                   # and may hold anything
        b[7] = math.nan
        index, w, key = C.route(z, b, score, groups, 2 if groups > 1 else 1, per, k, renorm, 1.0)
        got, gw = run_route(zo, z, b, k, score=score, groups=groups, top_groups=2 if groups > 1 else 1,
                            group_top=per, renormalise=renorm)
        assert torch.equal(got, index), (got != index).nonzero()
        C.within(gw, w, 120 * C.U * w.nan_to_num(nan=0.0).abs() + C.NORMAL, "weight")
        assert not (got == 4).any() and not (got == 7).any() and (got[0] == -1).all()
        assert not torch.isnan(gw[8]).any()


@pytest.mark.parametrize("slots,experts", ((0, 5), (1, 1), (1, 1024), (64, 3), (511, 8), (513, 1024), (2047, 16),
                                           (4096, 64), (5000, 60), (20000, 1024), (70001, 256), (600000, 2),
                                           (1100000, 7)))
def test_route_order(zo, slots, experts):
    g = C.rng(29, slots, experts)
    index = torch.randint(-1 if slots % 2 else 0, experts, (slots,), generator=g, dtype=torch.int32)
    if slots > 600:
        index[100:400] = experts // 2      # a run of one expert
        index[400] = experts               # outside: no expert
        index[401] = -2 ** 31
    oo, od = Out(1, experts + 1, torch.int32), Out(1, slots, torch.int32)
    n = zo.zero_route_workspace(slots, experts)
    assert n <= 1024 * (experts + 1)
    room = Out(1, n, torch.int32)
    zo.zero_route_order(index.cuda(), experts, oo.view[0], od.view[0], room.view[0])
    torch.cuda.synchronize()
    offsets, order = C.order(index, experts)
    assert oo.view[0].tolist() == offsets and od.view[0].tolist() == order
    assert oo.guards_intact() and od.guards_intact() and room.guards_intact()


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
@pytest.mark.parametrize("rows,experts,k", ((1, 1, 1), (3, 7, 7), (70, 64, 6), (33, 60, 4), (40, 256, 8), (9, 1023, 33),
                                            (5, 1024, 64), (130, 8, 2)))
def test_route_backward(zo, rows, experts, k, score, dtype):
    for renorm, pad in ((True, 0), (False, 5)):
        z, b = route_inputs(rows, experts, dtype, 31, True, grid=False)
        if experts > 8:
            b[3] = -math.inf
            z[0, 3] = math.nan
            z[0, 5:] = -math.inf
        g = C.rng(37, rows, experts)
        index, _, _ = C.route(z, b, score, 1, 1, 1, k, renorm, 1.0)
        dw = C.normal(g, rows, k).float()
        dw[index < 0] = math.nan  # not looked at
        want, size = C.route_backward(z, b, index, dw.nan_to_num(), score, renorm, 2.5)
        o = Out(rows, experts, dtype, pad)
        zd, id_, dd = put(z, pad), index.int().cuda(), dw.cuda()
        kw = dict(score=score, bias=b.cuda(), renormalise=renorm, scale=2.5)
        zo.zero_route_backward(zd, id_, dd, o.view, **kw)
        torch.cuda.synchronize()
        assert o.guards_intact()
        C.within(o.view, want, C.rounded(150 * C.U * size + C.NORMAL, want, dtype), "dlogits")
        mine = zd.clone()
        zo.zero_route_backward(mine, id_, dd, mine, **kw)
        assert torch.equal(mine, o.view)


@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
@pytest.mark.parametrize("renorm", (True, False))
def test_route_gradient_against_differences(zo, score, renorm):
    """Central differences of the fp32 weights: step 2^-6; the third derivative's term is under 2e-4, rounding
    under 2^-24 * 4 * 2^6."""
    g = C.rng(41)
    z, dw = C.normal(g, 2, 12).float(), C.normal(g, 2, 4).float()
    index, w = torch.empty(2, 4, dtype=torch.int32, device="cuda"), torch.empty(2, 4, device="cuda")
    zo.zero_route(z.cuda(), index, w, score=score, renormalise=renorm)
    d = torch.empty(2, 12, device="cuda")
    zo.zero_route_backward(z.cuda(), index, dw.cuda(), d, score=score, renormalise=renorm)
    at, step = index.cpu().long(), 2.0 ** -6
    for r in range(2):
        for c in range(12):
            both = []
            for s in (step, -step):
                zs = z.double()
                zs[r, c] += s
                ws = C.weights(zs, torch.zeros_like(z, dtype=torch.bool), at, score, renorm, 1.0)
                both.append((ws * dw.double()).sum())
            assert abs(float((both[0] - both[1]) / (2 * step)) - d[r, c].item()) < 5e-4


# --- distillation -------------------------------------------------------------------

def distill_inputs(rows, vocab, k, dtype, tdtype, seed):
    g = C.rng(seed, rows, vocab, k)
    z = C.normal(g, rows, vocab, std=2.0)
    index = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]) if k else None
    teacher = C.normal(g, rows, k, std=2.0) + 8 if k else None
    label = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    if k:
        z.scatter_add_(1, index, C.normal(g, rows, k) + 5)
        same = torch.rand(rows, generator=g) < 0.5
        label = torch.where(same, index[:, 0].int(), label)
        index = index.int()
        if k > 2:
            index[:, 1][torch.rand(rows, generator=g) < 0.3] = -1
    weight = torch.rand(rows, generator=g).float() + 0.5
    if rows > 2:
        weight[1] = 0.0
        label[2] = -1
    return z.to(dtype), index, teacher.to(tdtype) if k else None, label, weight


def dev(t):
    return None if t is None else t.cuda()


def check_distill(zo, z, index, teacher, label, weight, soft=1.0, hard=0.5, tau=2.0, scale=1024.0, pad=0, lead=0):
    rows, vocab = z.shape
    dtype = z.dtype
    loss, lb, g, gb = C.distill(z, index, teacher, label, soft, hard, tau, weight, scale)
    limit = C.rounded(gb, g, dtype)
    if dtype == F16:  # what rounds past the largest value is inf
        g = torch.where(g.abs() >= 65520, torch.sign(g) * math.inf, g)
    kw = dict(labels=dev(label), soft=soft, hard=hard, temperature=tau, row_weight=dev(weight))
    zd, id_, td = put(z, pad, lead), dev(index), dev(teacher)
    ol, og = Out(1, rows, F32), Out(rows, vocab, dtype, pad, lead)
    zo.zero_distill_step(zd, id_, td, ol.view[0], og.view, grad_scale=scale, **kw)
    torch.cuda.synchronize()
    assert ol.guards_intact() and og.guards_intact()
    C.within(ol.view[0], loss, lb, "loss")
    C.within(og.view, g, limit, "dlogits")
    # in place: the same bits
    mine = Out(rows, vocab, dtype, pad, lead)
    mine.view.copy_(z)
    zo.zero_distill_step(mine.view, id_, td, ol.view[0], mine.view, grad_scale=scale, **kw)
    assert mine.guards_intact() and torch.equal(mine.view.contiguous().view(torch.uint8),
                                                og.view.contiguous().view(torch.uint8))
    # the loss, then the gradient from its statistics and the losses' own gradient
    o2, og2, st = Out(1, rows, F32), Out(rows, vocab, dtype, pad, lead), Out(rows, 3, F32)
    zo.zero_distill_loss(zd, id_, td, o2.view[0], stats=st.view, **kw)
    C.within(o2.view[0], loss, lb, "loss alone")
    up = torch.rand(rows, generator=C.rng(3, rows)).float() + 0.5
    zo.zero_distill_backward(zd, id_, td, st.view, og2.view, dloss=dev(up), grad_scale=scale, **kw)
    torch.cuda.synchronize()
    assert o2.guards_intact() and og2.guards_intact() and st.guards_intact()
    _, _, g2, gb2 = C.distill(z, index, teacher, label, soft, hard, tau, weight, scale, up)
    if dtype == F16:
        g2 = torch.where(g2.abs() >= 65520, torch.sign(g2) * math.inf, g2)
    C.within(og2.view, g2, C.rounded(gb2, g2.nan_to_num(posinf=0.0, neginf=0.0), dtype), "dlogits of the backward")


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,vocab,k", ((1, 1, 1), (3, 5, 2), (4, 63, 8), (5, 1000, 16), (3, 2048, 128), (4, 2049, 3),
                                          (3, 4100, 64), (3, 8192, 33), (2, 12345, 1024), (3, 20000, 7), (2, 50257, 64),
                                          (2, 70001, 200), (2, 131072, 128), (1, 200003, 64)))
def test_distill(zo, rows, vocab, k, dtype):
    tdtype = C.TYPES[(rows + vocab + k) % 3]
    check_distill(zo, *distill_inputs(rows, vocab, k, dtype, tdtype, 43), hard=0.5 if k % 2 == 0 else 0.0,
                  tau=(1.0, 2.0, 1.5)[vocab % 3])


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("pad,lead", ((0, 1), (1, 0), (47, 3)))
def test_distill_strides(zo, pad, lead, dtype):
    for vocab in (37, 1001, 9000):
        check_distill(zo, *distill_inputs(5, vocab, 9, dtype, F32, 47), pad=pad, lead=lead)


@pytest.mark.parametrize("dtype", C.TYPES)
def test_distill_terms(zo, dtype):
    z, index, teacher, label, weight = distill_inputs(6, 777, 12, dtype, dtype, 53)
    check_distill(zo, z, None, None, label, weight, hard=1.0, tau=1.0)          # no teacher
    check_distill(zo, z, None, None, None, weight, hard=1.0)                    # nothing at all
    check_distill(zo, z, index, teacher, None, None, hard=1.0)                  # no labels, every row counts
    check_distill(zo, z, index, teacher, label, weight, soft=0.0, hard=1.0)     # the soft term switched off
    check_distill(zo, z, index, teacher, label, -weight, soft=0.7, hard=-0.3)   # signs as they come
    twice = index.clone()
    twice[:, 5] = twice[:, 0]                                                   # a token listed again, and thrice
    twice[:, 6] = twice[:, 0]
    twice[3, 7:] = twice[3, 2]
    check_distill(zo, z, twice, teacher, label, weight)
    far = index.clone()
    far[0], far[1, 3], far[2, 4] = -1, 777, 2 ** 31 - 1                         # absent, a whole row of them
    label[3], label[4] = 777, -2 ** 31
    check_distill(zo, z, far, teacher, label, weight)


def test_distill_tokens_far_apart(zo):
    """Tokens a multiple of the tables' sizes apart are told apart."""
    z, index, teacher, label, weight = distill_inputs(2, 140000, 6, F32, F32, 59)
    index[:, :4] = torch.tensor([5, 65541, 131077, 70000], dtype=torch.int32)
    label[:] = torch.tensor([65541, 6], dtype=torch.int32)
    check_distill(zo, z, index, teacher, label, weight)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("vocab", (300, 5000, 140000))
def test_distill_crowded(zo, dtype, vocab):
    """Every token of the first vectors is listed, the label among them."""
    z, index, teacher, label, weight = distill_inputs(3, vocab, 40, dtype, F32, 60)
    index[:] = torch.stack([torch.randperm(40, generator=C.rng(5, i)) for i in range(3)]).int()
    label[:] = torch.tensor([0, 39, 17], dtype=torch.int32)
    for lead in (0, 5):
        check_distill(zo, z, index, teacher, label, weight, lead=lead)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("vocab", (300, 5000, 140000))
def test_distill_masks(zo, dtype, vocab):
    z, index, teacher, label, weight = distill_inputs(10, vocab, 8, dtype, dtype, 61)
    weight[:] = 1.0
    label[:] = torch.arange(10, dtype=torch.int32)
    index[:] = torch.arange(8, dtype=torch.int32) * 3
    low = torch.finfo(dtype).min
    z[0] = -math.inf                       # no token: NaN
    z[1] = low                             # all at the lowest value: uniform
    z[2, 30:] = -math.inf                  # a mask that leaves 30
    z[3, 30:] = low
    z[4, 7] = math.nan
    z[5, 7] = math.inf
    z[6, index[6, 2].item()] = -math.inf   # the teacher wants what the student excludes: loss inf
    teacher[7, 1:] = -math.inf             # one entry
    teacher[8] = -math.inf                 # none
    weight[9] = 0.0                        # a row that is not looked at may hold anything
    z[9] = math.nan
    teacher[9] = math.nan
    check_distill(zo, z, index, teacher, label, weight, tau=2.0)
    check_distill(zo, z, index, teacher, None, weight, tau=1.0)
    teacher[1] = math.nan                  # a broken teacher shows
    loss = torch.empty(10, device="cuda")
    zo.zero_distill_loss(z.cuda(), index.cuda(), teacher.cuda(), loss, row_weight=weight.cuda())
    assert math.isnan(loss[1].item()) and loss[9].item() == 0


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tau", (1e-6, 1e-3, 50.0))
def test_distill_temperatures(zo, dtype, tau):
    """Far from 1 on both sides: a softmax that takes the largest alone, and an even one."""
    for vocab in (700, 9000):
        check_distill(zo, *distill_inputs(4, vocab, 10, dtype, dtype, 63), hard=0.25, tau=tau)


def test_distill_overflow_reaches_the_shard_step(zo):
    """A loss scale that takes the gradient past binary16 gives inf, on which the shard step skips."""
    from paper_1910_02054_amd import binding as zb
    z, index, teacher, label, weight = (dev(t) for t in distill_inputs(4, 100, 5, F16, F16, 67))
    n = z.numel()
    master, m, v = (torch.full((n,), 0.5, device="cuda") for _ in range(3))
    p16, g = torch.zeros(n, dtype=F16, device="cuda"), torch.empty_like(z)
    loss = torch.empty(4, device="cuda")
    flags = []
    for scale in (2.0 ** 24, 2.0 ** 10):
        zo.zero_distill_step(z, index, teacher, loss, g, row_weight=weight, grad_scale=scale)
        flags.append(zb.zero_shard_step(g.view(-1), master, m, v, p16, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, scale, 1.0))
    assert flags == [1, 0] and torch.isinf(g).sum() == 0


def test_distill_no_rows(zo):
    z = torch.empty(0, 64, dtype=F16, device="cuda")
    zo.zero_distill_step(z, torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda"),
                         torch.empty(0, device="cuda"), torch.empty_like(z))


def test_distill_gradient_against_differences(zo):
    """Central differences of the fp32 loss: step 2^-5, whose third-derivative term is under 1e-3 and whose
    rounding is under 20 * 2^-24 * 2^5."""
    z, index, teacher, label, _ = distill_inputs(2, 30, 6, F32, F32, 71)
    loss, g = torch.empty(2, device="cuda"), torch.empty(2, 30, device="cuda")
    args, kw = (dev(index), dev(teacher)), dict(labels=dev(label), hard=0.5, temperature=1.5)
    zo.zero_distill_step(z.cuda(), *args, loss, g, **kw)
    step = 2.0 ** -5
    for r in range(2):
        for c in range(0, 30, 3):
            both = []
            for s in (step, -step):
                zs = z.clone()
                zs[r, c] += s
                zo.zero_distill_loss(zs.cuda(), *args, loss, **kw)
                both.append(loss.cpu().double().sum())
            assert abs(float((both[0] - both[1]) / (2 * step)) - g[r, c].item()) < 2e-3


# --- what only a device can refuse ---------------------------------------------------

def test_arrays_outside_their_allocations_are_refused(zo):
    """A size that overruns an array's allocation and memory that the device cannot reach are refused before a launch."""
    x = torch.zeros(4, 256, dtype=F16, device="cuda")
    w, y = torch.ones(256, dtype=F16, device="cuda"), torch.zeros_like(x)
    host = torch.zeros(4, 256, dtype=F16)

    def call(rows, px, py):
        return zo._lib.zero_rms_norm(zo.RMS_NORM_ARGS.pack(1, 0, rows, 256, 1e-6, px, 256, 0, 256, w.data_ptr(), 0, 256, py,
                                                          256, 0, 256, 0, 0), zo._on(None))

    assert call(4, x.data_ptr(), y.data_ptr()) == 0
    # more rows than the device has memory for (torch's own allocations may be longer than a tensor)
    assert call(1 << 30, x.data_ptr(), x.data_ptr()) == -1
    said = zo._lib.zero_last_error().decode()
    assert "overruns its allocation" in said or "weight and y overlap" in said, said  # weight may lie in the span
    assert call(4, host.data_ptr(), y.data_ptr()) == -1
    assert "GPU-accessible" in zo._lib.zero_last_error().decode()
    with pytest.raises(zo.ZeroError) as e:
        zo.zero_rms_norm(x, w, -1.0, y=y)
    assert e.value.code == -1 and "eps" in str(e.value)
    with pytest.raises(ValueError):
        zo.zero_rms_norm(x, w, 1e-6, y=torch.zeros(4, 255, dtype=F16, device="cuda"))
    with pytest.raises(ValueError):
        zo.zero_rms_norm(x.t().contiguous().t(), w, 1e-6, y=y)
    with pytest.raises(TypeError):
        zo.zero_rms_norm(x, w.float(), 1e-6, y=y)
    with pytest.raises(TypeError):
        zo.zero_rms_norm(x, w, 1e-6, y=host)
    with pytest.raises(zo.ZeroError):  # rows that overlap the next ones
        zo.zero_rms_norm(torch.as_strided(x, (3, 256), (100, 1)), w, 1e-6, y=torch.zeros(3, 256, dtype=F16, device="cuda"))
    torch.cuda.synchronize()


# --- streams, graphs, sizes ---------------------------------------------------------

def all_calls(zo, seed, stream=None):
    """Every operator once on inputs of `seed`; returns a function that enqueues the calls and the outputs."""
    g = C.rng(seed)
    x, r = (C.normal(g, 70, 384).to(F16).cuda() for _ in range(2))
    w = torch.ones(384, dtype=F16, device="cuda")
    h, y, dx, q = (torch.zeros_like(x) for _ in range(4))
    q8, sc = torch.zeros(70, 384, dtype=torch.uint8, device="cuda"), torch.zeros(70, 3, device="cuda")
    rstd, dw = torch.zeros(70, device="cuda"), torch.zeros_like(w)
    room = torch.empty(zo.zero_rms_norm_workspace(70, 384), device="cuda")
    z, b = route_inputs(900, 64, F32, seed, True)
    z, b = z.cuda(), b.cuda()
    index, wt = torch.zeros(900, 6, dtype=torch.int32, device="cuda"), torch.zeros(900, 6, device="cuda")
    offsets = torch.zeros(65, dtype=torch.int32, device="cuda")
    order = torch.zeros(5400, dtype=torch.int32, device="cuda")
    iroom = torch.empty(zo.zero_route_workspace(5400, 64), dtype=torch.int32, device="cuda")
    dl = torch.zeros_like(z)
    s, idx, t, label, weight = (dev(a) for a in distill_inputs(9, 3001, 16, BF16, F32, seed))
    loss, loss2, ds, ds2 = (torch.zeros(9, device="cuda"), torch.zeros(9, device="cuda"), torch.zeros_like(s),
                            torch.zeros_like(s))
    st = torch.zeros(9, 3, device="cuda")
    kw = dict(labels=label, hard=0.5, temperature=2.0, row_weight=weight, stream=stream)

    def go():
        zo.zero_rms_norm(x, w, 1e-6, residual=r, h=h, y=y, q8=q8, scale=sc, group=128, rstd=rstd, stream=stream)
        zo.zero_rms_norm_backward(y, h, w, rstd, dx, dw, room, dh=r, stream=stream)
        zo.zero_route(z, index, wt, score="sigmoid", bias=b, stream=stream)
        zo.zero_route_order(index, 64, offsets, order, iroom, stream=stream)
        zo.zero_route_backward(z, index, wt, dl, score="sigmoid", bias=b, stream=stream)
        zo.zero_distill_step(s, idx, t, loss, ds, grad_scale=64.0, **kw)
        zo.zero_distill_loss(s, idx, t, loss2, stats=st, **kw)
        zo.zero_distill_backward(s, idx, t, st, ds2, grad_scale=64.0, **kw)

    return go, (h, y, q8, sc, rstd, dx, dw, index, wt, offsets, order, dl, loss, ds, loss2, st, ds2), (x, z, s)


def bits(ts):
    return [t.clone().view(torch.uint8) for t in ts]


def test_operators_on_another_stream(zo):
    go, outs, _ = all_calls(zo, 73)
    go()
    want = bits(outs)
    side = torch.cuda.Stream()
    go2, outs2, _ = all_calls(zo, 73, stream=side)
    side.wait_stream(torch.cuda.current_stream())
    go2()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, bits(outs2)))


def test_operators_in_a_graph(zo):
    go, outs, ins = all_calls(zo, 79)
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for turn in range(3):
        for t in ins:  # new inputs for every replay
            t.mul_(0.75)
        go()
        want = bits(outs)
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, bits(outs))), turn


def test_more_rows_than_one_launch(zo):
    """Rows past the workgroups of one launch (2^20, of 16 short rows, of one router's token or one distilled row)."""
    n = (1 << 20) + 3
    x = torch.randn(n, 8, device="cuda", dtype=F16)
    z = x.clone()
    loss, g = torch.empty(n, device="cuda"), torch.empty_like(z)
    idx = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    zo.zero_distill_step(z, idx, torch.ones(n, 1, device="cuda"), loss, g)
    want = torch.softmax(z.float(), 1)
    want[:, 0] -= 1
    assert (g.float() - want).abs().max() < 2e-3
    big = torch.randn(16 * n, 8, device="cuda", dtype=F16)
    y = torch.zeros_like(big)
    zo.zero_rms_norm(big, torch.ones(8, device="cuda", dtype=F16), 1e-6, y=y)
    f = big.float()
    assert (y.float() - f / (f.square().mean(1, keepdim=True) + 1e-6).sqrt()).abs().max() < 4e-3
    m = 32 * (1 << 20) + 40
    z = torch.randn(m, 4, device="cuda", dtype=F16)
    index, w = torch.empty(m, 1, dtype=torch.int32, device="cuda"), torch.empty(m, 1, device="cuda")
    zo.zero_route(z, index, w, renormalise=False)
    assert torch.equal(z.gather(1, index.long()), z.amax(1, keepdim=True))
    d = torch.empty_like(z)
    zo.zero_route_backward(z, index, torch.ones_like(w), d, score="sigmoid", renormalise=False)
    s = torch.sigmoid(z.gather(1, index.long()).float())
    assert (d.gather(1, index.long()).float() - s * (1 - s)).abs().max() < 2e-3
    assert (d != 0).sum() <= m


def test_offsets_past_32_bits(zo):
    """Rows far apart: the last row of each matrix lies past 2^32 elements from the first."""
    ld, rows = (1 << 31) + 64, 3
    buf = torch.zeros((rows - 1) * ld + 2048, dtype=F16, device="cuda")
    x = torch.as_strided(buf, (rows, 1024), (ld, 1))
    x.copy_(torch.randn(rows, 1024, device="cuda"))
    y = torch.as_strided(buf, (rows, 1024), (ld, 1), 1024)
    w = torch.ones(1024, device="cuda", dtype=F16)
    zo.zero_rms_norm(x, w, 1e-6, y=y)
    f = x.float()
    assert (y.float() - f / (f.square().mean(1, keepdim=True) + 1e-6).sqrt()).abs().max() < 4e-3
    idx = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    loss = torch.empty(rows, device="cuda")
    zo.zero_distill_step(x, idx, torch.ones(rows, 1, device="cuda"), loss, y)
    want = torch.softmax(f, 1)
    want[:, 0] -= 1
    assert (y.float() - want).abs().max() < 1e-3
