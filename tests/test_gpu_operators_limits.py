"""The training operators on the GPU at the ends of their types' ranges, and at every shape of their kernels that the
sizes of test_gpu_operators.py do not reach."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_checks as C  # noqa: E402
import test_gpu_operators as G  # noqa: E402
from test_gpu_operators import Out, put  # noqa: E402

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def zo():
    from paper_1910_02054_amd import operators
    assert torch.cuda.is_available()
    return operators


# --- e4m3 codes -------------------------------------------------------------------

def run_e4m3(zo, h, w, group, eps):
    """(codes, scale, rstd) of the rows h, on the CPU."""
    rows, cols = h.shape
    q = Out(rows, cols, torch.uint8)
    scale, rstd = Out(rows, -(-cols // group) if group else 1, F32), Out(rows, 1, F32)
    zo.zero_rms_norm(put(h), w.cuda(), eps, q8=q.view, scale=scale.view, group=group, rstd=rstd.view)
    torch.cuda.synchronize()
    assert q.guards_intact() and scale.guards_intact() and rstd.guards_intact()
    return q.view.cpu(), scale.view.cpu(), rstd.view.cpu()


def e4m3(q):
    return q.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,cols,group", ((5, 100, 0), (300, 1603, 64), (257, 4096, 128), (9, 8200, 0)))
def test_codes_are_of_the_quotient(zo, rows, cols, group, dtype):
    """y's fp32 value is two products of the row, the rstd that the call returned and the weight, and the scale is
    returned too, so the code of fl(y / scale) has no room: not where 8-bit mantissas make the quotient a tie
    either."""
    g = C.rng(83, rows, cols)
    h, w = C.normal(g, rows, cols).to(dtype), (1 + 0.1 * C.normal(g, cols)).to(dtype)
    q, scale, rstd = run_e4m3(zo, h, w, group, 1e-6)
    y = h.float() * rstd * w.float()
    assert torch.equal(scale, torch.stack([p.abs().amax(1) for p in y.split(group or cols, 1)], 1) / 448.0)
    assert torch.equal(q, e4m3(y / C.spread(scale, cols, group)))


@pytest.mark.parametrize("exponent", (-126, -110, -100, -81, -79, 0, 60, 126))
def test_codes_beside_the_ties(zo, exponent):
    """Rows of ones have rstd 1, so y is the weight: each midpoint of two neighbouring codes times the scale, and its
    three neighbours on both sides, under 40 scales."""
    g = C.rng(89, exponent + 200)
    v = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    ties = (v[1:] + v[:-1]) / 2
    for _ in range(40):
        top = (torch.rand(1, generator=g) + 1.0) * 2.0 ** exponent
        t = top.clamp(min=2.0 ** -100) / 448.0
        w = torch.cat([top] + [(ties * t).view(torch.int32).add(k).view(F32) for k in range(-3, 4)])
        w = torch.where(w <= top, w, top) * torch.where(torch.rand(w.shape, generator=g) < 0.5, -1.0, 1.0)
        q, scale, rstd = run_e4m3(zo, torch.ones(1, w.numel()), w, 0, 0.0)
        assert rstd.item() == 1.0 and scale.item() == t.item()
        assert torch.equal(q[0], e4m3(w / t))


# --- routing: saturated scores --------------------------------------------------------

@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("renorm", (False, True))
def test_route_backward_of_saturated_scores(zo, renorm, dtype):
    """The sigmoid's slope s (1 - s) where s is near 1: a few units of the slope itself, as an exponential, two sums and
    two quotients leave, not of s."""
    values = torch.tensor([-60.0, -40.0, -20.0, -16.0, -12.0, -5.0, 0.0, 5.0, 9.0, 12.0, 14.0, 16.0, 17.0, 18.0, 20.0,
                           30.0, 40.0, 60.0, 80.0])
    g = C.rng(97)
    rows, experts, k = 64, 24, 6
    z = values[torch.randint(0, len(values), (rows, experts), generator=g)].to(dtype)
    index = torch.stack([torch.randperm(experts, generator=g)[:k] for _ in range(rows)])
    dw = C.normal(g, rows, k).float()
    zc, d = z.double().gather(1, index), dw.double() * 2.5
    s, slope = torch.sigmoid(zc), torch.sigmoid(zc) * torch.sigmoid(-zc)
    t, size = d, d.abs()
    if renorm:
        total = s.sum(1, keepdim=True)
        t = (d - (d * s).sum(1, keepdim=True) / total) / total
        size = (d.abs() + (d * s).abs().sum(1, keepdim=True) / total) / total
    want = torch.zeros(rows, experts, dtype=torch.float64).scatter_add(1, index, t * slope)
    units = 12 if not renorm else 60    # two sums of six terms, two quotients and a difference more
    bound = torch.zeros_like(want).scatter_add(1, index, units * C.U * size * slope)
    out = Out(rows, experts, dtype)
    zo.zero_route_backward(put(z), index.int().cuda(), dw.cuda(), out.view, score="sigmoid", renormalise=renorm,
                           scale=2.5)
    torch.cuda.synchronize()
    assert out.guards_intact()
    C.within(out.view, want, C.rounded(bound, want, dtype), "dlogits")


# --- distillation: masks and temperatures ------------------------------------------------

def run_loss(zo, z, index, teacher, labels=None, **kw):
    """The losses [2, rows] by the step and by the call of their own."""
    both = torch.empty(2, z.shape[0], device="cuda")
    args = (put(z), None if index is None else index.cuda(), None if teacher is None else teacher.cuda())
    kw["labels"] = None if labels is None else labels.cuda()
    zo.zero_distill_step(*args, both[0], torch.empty(z.shape, dtype=z.dtype, device="cuda"), **kw)
    zo.zero_distill_loss(*args, both[1], **kw)
    return both.cpu()


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("vocab", (300, 5000, 140000))
@pytest.mark.parametrize("tau", (1.0, 2.0, 1.5))
def test_distill_wants_a_token_at_the_lowest_value(zo, tau, vocab, dtype):
    """A student masked by its type's lowest value, not by -inf, where the teacher or the label wants the token: the loss is
    the gap times the token's share, which fp32 holds.  Each loss is one product of the largest term, a few units."""
    g = C.rng(101, vocab)
    z = C.normal(g, 4, vocab)
    index = torch.tensor([[3, 9, 20]] * 4, dtype=torch.int32)
    teacher = torch.tensor([[1.0, 2.0, 0.5]] * 4)
    labels = torch.tensor([5, 7, 50, 60], dtype=torch.int32)
    low = torch.finfo(dtype).min
    z[0, 9] = low            # the teacher's largest
    z[1, 7] = low            # the label
    z[2, :40] = low          # every token of the list
    z = z.to(dtype)
    soft, hard = 0.05, 0.25
    loss = run_loss(zo, z, index, teacher, labels, soft=soft, hard=hard, temperature=tau)
    want, _, _, _ = C.distill(z, index, teacher, labels, soft, hard, tau, None, 1.0)
    assert torch.isfinite(want.float()).all()
    C.within(loss, want.expand(2, -1), 60 * C.U * want.abs() + 60 * C.U * 20, "loss")


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tau", (1e-30, 1e-25, 1e-22, 1e-19, 1e-12, 1e-6))
def test_distill_low_temperatures(zo, tau, dtype):
    """Next to nothing, the teacher's largest takes all, the student's too: the loss is soft tau times the gap between its
    maximum and the logit of the teacher's token."""
    g = C.rng(103)
    for vocab in (700, 9000):
        z, teacher = (C.normal(g, 5, vocab) * 4).to(dtype), C.normal(g, 5, 6)
        index = torch.stack([torch.randperm(vocab, generator=g)[:6] for _ in range(5)]).int()
        at = index.gather(1, teacher.float().argmax(1, keepdim=True)).long()
        want = 0.7 * tau * (z.double().amax(1) - z.double().gather(1, at)[:, 0])
        loss = run_loss(zo, z, index, teacher.float(), soft=0.7, temperature=tau)
        # where the two agree, what the two sums' logarithms leave of tau^2
        C.within(loss, want.expand(2, -1), 12 * C.U * want + 60 * C.U * tau ** 2 + C.TINY[F32], "loss")


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tau", (1e3, 1e10, 1e18))
def test_distill_high_temperatures(zo, tau, dtype):
    """An even student against an even list of a part of the vocabulary: soft tau^2 ln(vocab / entries) in the main."""
    g = C.rng(107)
    z, teacher = C.normal(g, 5, 4000).to(dtype), C.normal(g, 5, 10).float()
    index = torch.stack([torch.randperm(4000, generator=g)[:10] for _ in range(5)]).int()
    want, _, _, _ = C.distill(z, index, teacher, None, 0.7, 0.0, tau, None, 1.0)
    loss = run_loss(zo, z, index, teacher, soft=0.7, temperature=tau)
    C.within(loss, want.expand(2, -1), 60 * C.U * want, "loss")


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tau", (1e20, 1e30))
def test_distill_whole_list_at_any_temperature(zo, tau, dtype):
    """A list of the whole vocabulary, on which the student agrees with the teacher: nothing is left but rounding, of which
    the header says that it grows with tau^2; but never a NaN."""
    z = torch.tensor([[1.0, 2.0, 0.5, -1.0]] * 3).to(dtype)
    index = torch.arange(4, dtype=torch.int32).repeat(3, 1)
    loss = run_loss(zo, z, index, z.float(), temperature=tau)
    assert not loss.isnan().any()


# --- norm: the ends of the range ----------------------------------------------------------

WIDE = (3, 8, 64, 100, 200, 512, 1603, 4100, 8200, 20000, 32768)


@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("rows", (9, 300))
@pytest.mark.parametrize("cols", WIDE)
def test_norm_of_the_largest_and_the_smallest(zo, cols, rows, dtype):
    """Rows whose squares leave fp32's range on either side, among ordinary ones (rows that share a wave among them):
    rstd and y are as finite as the formula's.  eps is 0, so that nothing hides the small ones."""
    if rows * cols > 3000000:
        rows = 258
    g = C.rng(109, rows, cols)
    x, w = C.normal(g, rows, cols), (1 + 0.1 * C.normal(g, cols)).to(dtype)
    big = torch.finfo(dtype).max
    x[0] = big
    x[1, cols // 2] = -big
    x[2] *= 1e19
    x[4] *= 1e-25
    x[5] = 2.0 ** -120
    x[6] *= 1e30
    x[6, 0] = 1e-30
    x[rows - 1] = -big
    x = x.to(dtype)
    rstd, y = C.rms_norm(x, w, 0.0)
    oy, orr = Out(rows, cols, dtype), Out(rows, 1, F32)
    oq, osc = Out(rows, cols, torch.uint8), Out(rows, 1, F32)
    zo.zero_rms_norm(put(x), w.cuda(), 0.0, y=oy.view, rstd=orr.view, q8=oq.view, scale=osc.view)
    torch.cuda.synchronize()
    assert oy.guards_intact() and orr.guards_intact() and oq.guards_intact() and osc.guards_intact()
    # a rstd below fp32's normal range is rounded to a multiple of 2^-149
    off = (C.ROOT + 4 * C.U) * rstd + C.TINY[F32]
    C.within(orr.view[:, 0], rstd, off, "rstd")
    # and so are the two products of y
    off = (C.ROOT + 8 * C.U + C.TINY[F32] / rstd)[:, None] * y.abs() + 4 * C.TINY[F32]
    C.within(oy.view, y, C.rounded(off, y, dtype), "y")
    C.check_e4m3(oq.view.contiguous(), y, 0, "q8")
    # the backward of the same rows
    dy = C.normal(g, rows, cols).to(dtype)
    r32 = orr.view[:, 0].contiguous()
    dx, dw, bx, bw = C.rms_norm_backward(dy, x, w, r32.cpu(), None)
    ox, ow = Out(rows, cols, dtype), Out(1, cols, dtype)
    room = Out(1, zo.zero_rms_norm_workspace(rows, cols), F32)
    zo.zero_rms_norm_backward(put(dy), put(x), w.cuda(), r32, ox.view, ow.view[0], room.view[0])
    torch.cuda.synchronize()
    assert ox.guards_intact() and ow.guards_intact() and room.guards_intact()
    # products below fp32's normal range each lose up to 2^-150
    C.within(ox.view, dx, C.rounded(bx + 8 * C.TINY[F32], dx, dtype), "dx")
    C.within(ow.view[0], dw, C.rounded(bw, dw, dtype), "dw")


def test_norm_of_any_eps(zo):
    """eps is a double: one below or above fp32's range counts as what it is."""
    x = torch.zeros(3, 100)
    x[1] = 1e-30
    x[2] = 3.0
    w = torch.ones(100)
    for eps in (0.0, 1e-300, 1e-61, 1e-40, 1e-20, 1e20, 1e50, 1e70, 1e100):
        y, rstd = torch.empty(3, 100, device="cuda"), torch.empty(3, device="cuda")
        zo.zero_rms_norm(x.cuda(), w.cuda(), eps, y=y, rstd=rstd)
        rd, yd = C.rms_norm(x, w, eps)
        want, wy = rd.float().double(), (x.double() * rd.float().double()[:, None])
        C.within(rstd, want, (C.ROOT + 4 * C.U) * rd.clamp(max=3.4e38) + 2 * C.TINY[F32], "rstd")
        C.within(y, wy, C.rounded((C.ROOT + 8 * C.U) * wy.abs().nan_to_num(posinf=0.0), wy, F32), "y")


# --- shapes of the kernels that other tests' sizes do not reach ------------------------------

@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows,cols", ((259, 1603), (258, 2041), (261, 1021), (257, 4089), (257, 2045), (259, 1100),
                                       (258, 2048), (257, 4096), (300, 8200)))
def test_norm_of_many_rows(zo, rows, cols, dtype):
    """Above 256 rows, wide rows take four or two vectors a lane in place of a workgroup of 1024."""
    for group in (0, 32, 256):
        G.check_norm(zo, rows, cols, dtype, group)
    G.check_norm(zo, rows, cols, dtype, 64, residual=False, pad=5, lead=3)
    G.check_norm(zo, rows, cols, dtype, 128, pad=3, lead=1, in_place=True)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
@pytest.mark.parametrize("shape", ((33, 128, 8, 1, 1, 1), (9, 64, 12, 1, 1, 1), (9, 100, 20, 1, 1, 1),
                                   (9, 512, 33, 1, 1, 1), (70, 128, 8, 4, 2, 2), (19, 112, 16, 8, 4, 2)))
def test_route_of_middling_sizes(zo, shape, score, dtype):
    """16 lanes a token with 4 and 8 keys, 32 with 4, 64 with 8."""
    G.test_route(zo, shape, score, dtype)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("score", ("softmax", "sigmoid"))
@pytest.mark.parametrize("rows,experts,k", ((33, 128, 8), (9, 100, 20), (70, 72, 4)))
def test_route_backward_of_middling_sizes(zo, rows, experts, k, score, dtype):
    G.test_route_backward(zo, rows, experts, k, score, dtype)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("vocab,k", ((3001, 16), (32003, 33), (60001, 64), (100277, 100)))
def test_distill_of_more_vocabularies(zo, vocab, k, dtype):
    """Shapes between the sizes of test_distill: 16-bit rows of 13 vectors a thread, fp32 rows of 4, 10 and 16."""
    G.check_distill(zo, *G.distill_inputs(3, vocab, k, dtype, C.TYPES[vocab % 3], 113), tau=(1.0, 2.0, 1.5)[k % 3])


def test_offsets_past_32_bits_of_the_other_calls(zo):
    """As test_offsets_past_32_bits of test_gpu_operators.py, for the gradients, the routing and the loss alone: the same
    bits as from rows that lie close together."""
    ld, rows, cols = (1 << 31) + 64, 3, 512
    buf = torch.zeros((rows - 1) * ld + 4 * cols, dtype=F16, device="cuda")
    a, b, c, d = (torch.as_strided(buf, (rows, cols), (ld, 1), i * cols) for i in range(4))
    near = [torch.randn(rows, cols, device="cuda").to(F16) for _ in range(3)]
    for far, t in zip((a, b, c), near):
        far.copy_(t)
    w, rstd = torch.ones(cols, device="cuda", dtype=F16), torch.rand(rows, device="cuda") + 0.5
    room, dw, dw2, out = torch.empty(4 * cols, device="cuda"), w.clone(), w.clone(), torch.empty_like(near[0])
    zo.zero_rms_norm_backward(a, b, w, rstd, d, dw, room, dh=c)
    zo.zero_rms_norm_backward(near[0], near[1], w, rstd, out, dw2, room, dh=near[2])
    assert torch.equal(d, out) and torch.equal(dw, dw2)
    index, index2 = (torch.empty(rows, 6, dtype=torch.int32, device="cuda") for _ in range(2))
    weight, weight2 = (torch.empty(rows, 6, device="cuda") for _ in range(2))
    zo.zero_route(a, index, weight)
    zo.zero_route(near[0], index2, weight2)
    assert torch.equal(index, index2) and torch.equal(weight, weight2)
    for renorm in (True, False):
        zo.zero_route_backward(a, index, weight, d, renormalise=renorm)
        zo.zero_route_backward(near[0], index, weight, out, renormalise=renorm)
        assert torch.equal(d, out)
    idx, teacher = torch.arange(rows * 4, dtype=torch.int32, device="cuda").view(rows, 4), torch.rand(rows, 4, device="cuda")
    loss, loss2, st, st2 = (torch.empty(rows, n, device="cuda") for n in (1, 1, 3, 3))
    zo.zero_distill_loss(a, idx, teacher, loss, stats=st)
    zo.zero_distill_loss(near[0], idx, teacher, loss2, stats=st2)
    assert torch.equal(loss, loss2) and torch.equal(st, st2)
    zo.zero_distill_backward(a, idx, teacher, st, d)
    zo.zero_distill_backward(near[0], idx, teacher, st, out)
    assert torch.equal(d, out)
