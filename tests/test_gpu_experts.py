"""The experts' operators on the GPU against plain 64-bit implementations (expert_checks.py): sizes, layouts and types,
experts without rows, slots without experts, bad order entries, strides, and the whole path from the
router's choice to the gradients."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import expert_checks as E  # noqa: E402
import operator_checks as C  # noqa: E402
from test_gpu_operators import Out, put  # noqa: E402

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def zo():
    from paper_1910_02054_amd import operators
    assert torch.cuda.is_available()
    return operators


def run_product(zo, tokens, k, experts, cin, cout, dtype, x_slots=0, y_slots=0, transposed=False, pad=0, lead=0,
                none=0.0, only=None, seed=1, x=None, w=None):
    slots = tokens * k
    index, offsets, placed = E.choice(tokens, k, experts, seed, none, only)
    g = C.rng(seed, cin, cout)
    rows = slots // x_slots if x_slots > 1 else slots
    if x is None:
        x = C.normal(g, rows, cin).to(dtype)
    if w is None:
        w = (C.normal(g, experts, *((cout, cin) if transposed else (cin, cout))) * cin ** -0.5).to(dtype)
    want, bound, written = E.product(x, w, offsets, placed, x_slots, y_slots, transposed, slots)
    out = Out(slots, cout, dtype, pad, lead)
    dw = put(w.flatten(0, 1), pad, lead)
    zo.zero_expert_product(put(x, pad, lead), dw.unflatten(0, (experts, -1)), offsets.cuda(), out.view,
                           order=placed.cuda() if x_slots or y_slots else None, x_slots=x_slots, y_slots=y_slots,
                           transposed=transposed)
    torch.cuda.synchronize()
    assert out.guards_intact()
    assert (out.view.cpu()[~written].view(-1).view(torch.uint8) == 0xA5).all()  # left as they were
    C.within(out.view.cpu()[written], want[written], C.rounded(bound, want, dtype)[written], "y")
    return out.view


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,experts,cin,cout", (
    (1, 1, 1, 1, 1), (1, 2, 4, 8, 8), (3, 2, 5, 7, 9), (8, 6, 64, 128, 136), (40, 2, 3, 65, 129), (37, 3, 7, 200, 24),
    (130, 2, 2, 264, 264), (257, 2, 1, 96, 130), (300, 4, 2, 72, 264), (700, 2, 2, 136, 300), (1, 1, 1024, 64, 32)))
def test_product_sizes(zo, tokens, k, experts, cin, cout, dtype):
    for transposed in (False, True):
        run_product(zo, tokens, k, experts, cin, cout, dtype, transposed=transposed)
        run_product(zo, tokens, k, experts, cin, cout, dtype, k, 1, transposed, none=0.1, seed=2)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("x_slots,y_slots", ((0, 0), (0, 1), (1, 0), (1, 1), (3, 0), (3, 1)))
def test_product_layouts_and_strides(zo, x_slots, y_slots, dtype):
    for pad, lead in ((0, 0), (8, 0), (3, 1), (0, 2)):
        for transposed in (False, True):
            run_product(zo, 50, 3, 4, 104, 168, dtype, x_slots, y_slots, transposed, pad, lead, 0.05)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,only", ((900, [2]), (900, [0, 5]), (20, [5]), (150, [1])))
def test_product_of_few_of_the_experts(zo, tokens, only, dtype):
    run_product(zo, tokens, 2, 6, 80, 264, dtype, 2, 1, only=only)


def test_product_without_rows(zo):
    w = torch.zeros(3, 16, 8, dtype=F16, device="cuda")
    none = torch.empty(0, 16, dtype=F16, device="cuda")
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    zo.zero_expert_product(none, w, offsets, torch.empty(0, 8, dtype=F16, device="cuda"))
    out = Out(6, 8, F16)  # every slot without an expert
    zo.zero_expert_product(torch.ones(3, 16, dtype=F16, device="cuda"), w, offsets, out.view,
                           order=torch.full((6,), -1, dtype=torch.int32, device="cuda"), x_slots=2, y_slots=1)
    torch.cuda.synchronize()
    assert (out.raw == 0xA5).all()


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens", (10, 200, 1300))
def test_product_keeps_rows_and_experts_apart(zo, tokens, dtype):
    """A NaN or an infinity in one row of x reaches that row of y alone, one in an expert's weights that expert's
    rows and the columns it stands in."""
    index, offsets, placed = E.choice(tokens, 1, 3, 5)
    g = C.rng(9)
    x, w = C.normal(g, tokens, 72).to(dtype), C.normal(g, 3, 72, 40).to(dtype)
    x[3, 71], x[5, 0] = math.nan, math.inf
    w[1, 70, 11] = math.nan
    for transposed in (False, True):
        ww = w.transpose(1, 2).contiguous() if transposed else w
        out = Out(tokens, 40, dtype)
        zo.zero_expert_product(x.cuda(), ww.cuda(), offsets.cuda(), out.view, order=placed.cuda(), x_slots=1, y_slots=1,
                               transposed=transposed)
        y = out.view.cpu()
        assert torch.isnan(y[3]).all() and not torch.isfinite(y[5]).any()
        rest = [i for i in range(tokens) if i not in (3, 5)]
        hit = (index[rest, 0] == 1)
        assert torch.isnan(y[rest][hit][:, 11]).all()
        clean = y[rest].clone()
        clean[:, 11][hit] = 0
        assert torch.isfinite(clean).all()


@pytest.mark.parametrize("dtype", C.TYPES)
def test_bad_order_and_offsets_stay_inside(zo, dtype):
    """Entries of order that name no slot give rows of zeros where x is read and write none; offsets that leave
    [0, slots] end there, and those that fall have no rows."""
    tokens, k, cin, cout = 30, 2, 40, 24
    slots = tokens * k
    _, offsets, placed = E.choice(tokens, k, 4, 11)
    g = C.rng(13)
    x, w = C.normal(g, tokens, cin).to(dtype), C.normal(g, 4, cin, cout).to(dtype)
    bad = placed.clone()
    bad[5], bad[17], bad[40] = -1, slots, 2 ** 31 - 1
    y = Out(slots, cout, dtype)
    zo.zero_expert_product(x.cuda(), w.cuda(), offsets.cuda(), y.view, order=bad.cuda(), x_slots=2)
    want, bound, _ = E.product(x, w, offsets, placed, 2, 0, False, slots)
    want[[5, 17, 40]] = 0
    C.within(y.view, want, C.rounded(bound, want, dtype), "y")
    y = Out(slots, cout, dtype)
    zo.zero_expert_product(x.cuda(), w.cuda(), offsets.cuda(), y.view, order=bad.cuda(), x_slots=2, y_slots=1)
    torch.cuda.synchronize()
    assert y.guards_intact() and (y.view.view(torch.uint8).view(slots, -1).cpu() == 0xA5).all(1).sum() == 3
    dw, db = E.weight_backward(x, want.to(dtype), offsets, placed, 2, 0)
    got = Out(4 * cin, cout, dtype)
    dy = want.to(dtype)
    zo.zero_expert_weight_backward(x.cuda(), dy.cuda(), offsets.cuda(), got.view.unflatten(0, (4, cin)), order=bad.cuda(),
                                   x_slots=2)
    C.within(got.view.unflatten(0, (4, cin)), dw, C.rounded(db, dw, dtype), "dw")  # those rows of dy are 0
    far = torch.tensor([-7, 20, 10, 2 ** 31 - 1, slots], dtype=torch.int32)
    y = Out(slots, cout, dtype)
    zo.zero_expert_product(x.cuda(), w.cuda(), far.cuda(), y.view, order=placed.cuda(), x_slots=2)
    zo.zero_expert_weight_backward(x.cuda(), dy.cuda(), far.cuda(), got.view.unflatten(0, (4, cin)), order=placed.cuda(),
                                   x_slots=2)
    torch.cuda.synchronize()
    assert y.guards_intact() and got.guards_intact()
    rows = x[placed.long() // 2].double()
    one = rows[:20] @ w[0].double()
    C.within(y.view[:10], one[:10], C.rounded((cin + 8) * 2 * C.U * (rows[:10].abs() @ w[0].double().abs()), one[:10],
                                              dtype), "first run")
    assert (got.view.unflatten(0, (4, cin))[1] == 0).all()


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,experts,cin,cout", (
    (1, 1, 1, 1, 1), (2, 2, 4, 8, 8), (3, 2, 5, 7, 9), (8, 6, 64, 16, 24), (40, 2, 3, 65, 129), (130, 2, 2, 136, 264),
    (2100, 2, 2, 24, 40), (3000, 1, 3, 130, 17), (1, 1, 1024, 8, 8)))
def test_weight_backward_sizes(zo, tokens, k, experts, cin, cout, dtype):
    for x_slots, dy_slots, pad, lead, none in ((0, 0, 0, 0, 0.0), (k, 1, 8, 0, 0.1), (1, k, 3, 1, 0.1)):
        index, offsets, placed = E.choice(tokens, k, experts, 3, none)
        slots = tokens * k
        g = C.rng(7, cin, cout)
        x = C.normal(g, slots // x_slots if x_slots > 1 else slots, cin).to(dtype)
        dy = C.normal(g, slots // dy_slots if dy_slots > 1 else slots, cout).to(dtype)
        want, bound = E.weight_backward(x, dy, offsets, placed, x_slots, dy_slots)
        out = Out(experts * cin, cout, dtype, pad, lead)
        n = zo.zero_expert_workspace(slots, experts, cin, cout)
        room = Out(1, n, F32)
        args = (put(x, pad, lead), put(dy, pad, lead), offsets.cuda())
        kw = dict(order=placed.cuda() if x_slots or dy_slots else None, x_slots=x_slots, dy_slots=dy_slots)
        zo.zero_expert_weight_backward(*args, out.view.unflatten(0, (experts, cin)), room.view[0], **kw)
        torch.cuda.synchronize()
        assert out.guards_intact() and room.guards_intact()
        C.within(out.view.unflatten(0, (experts, cin)), want, C.rounded(bound, want, dtype), "dw")
        again = torch.empty(experts, cin, cout, dtype=dtype, device="cuda")
        zo.zero_expert_weight_backward(*args, again, room.view[0], **kw)
        assert torch.equal(again.view(-1, cout), out.view)


def test_weight_backward_without_rows(zo):
    dw = torch.full((3, 8, 16), 7.0, dtype=F16, device="cuda")
    zo.zero_expert_weight_backward(torch.empty(0, 8, dtype=F16, device="cuda"),
                                   torch.empty(0, 16, dtype=F16, device="cuda"),
                                   torch.zeros(4, dtype=torch.int32, device="cuda"), dw)
    assert (dw == 0).all()


@pytest.mark.parametrize("dtype", C.TYPES)
def test_weight_backward_keeps_experts_apart(zo, dtype):
    """A row that overflowed reaches its expert's gradient, in its column, and no other."""
    index, offsets, placed = E.choice(90, 2, 3, 5)
    g = C.rng(9)
    x, dy = C.normal(g, 90, 24).to(dtype), C.normal(g, 180, 16).to(dtype)
    dy[7, 3] = math.inf
    dw = torch.empty(3, 24, 16, dtype=dtype, device="cuda")
    zo.zero_expert_weight_backward(x.cuda(), dy.cuda(), offsets.cuda(), dw, order=placed.cuda(), x_slots=2, dy_slots=1)
    bad = ~torch.isfinite(dw.cpu())
    e = int(index.view(-1)[7])
    assert bad[e, :, 3].all() and bad.sum() == 24


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,cols,pad,lead,weighted,base", (
    (1, 1, 1, 0, 0, True, False), (5, 2, 7, 0, 1, True, True), (8, 6, 130, 3, 0, False, True), (33, 4, 1603, 0, 0, True, True),
    (70, 5, 264, 8, 0, True, False), (3, 64, 520, 0, 0, False, False), (129, 3, 4100, 0, 3, True, True),
    (2, 8, 32768, 0, 0, True, True)))
def test_mix(zo, tokens, k, cols, pad, lead, weighted, base, dtype):
    g = C.rng(21, tokens, k, cols)
    index = torch.randint(-1, 9, (tokens, k), generator=g).int()
    y, dout = C.normal(g, tokens * k, cols).to(dtype), C.normal(g, tokens, cols).to(dtype)
    y.view(tokens, k, cols)[index < 0] = math.nan   # not looked at
    b = C.normal(g, tokens, cols).to(dtype) if base else None
    w = C.normal(g, tokens, k).float() if weighted else None
    for experts in (0, 6):
        yy = y.clone()
        yy.view(tokens, k, cols)[~E.there(index, experts)] = math.nan
        want, bound = E.mix(yy, index, w, b, experts)
        out = Out(tokens, cols, dtype, pad, lead)
        zo.zero_expert_mix(put(yy, pad, lead), index.cuda(), out.view, weight=None if w is None else w.cuda(),
                           base=None if b is None else put(b, pad, lead), experts=experts)
        torch.cuda.synchronize()
        assert out.guards_intact()
        C.within(out.view, want, C.rounded(bound, want, dtype), "out")
        if base:  # in place
            mine = put(b, pad, lead)
            zo.zero_expert_mix(put(yy, pad, lead), index.cuda(), mine, weight=None if w is None else w.cuda(), base=mine,
                               experts=experts)
            assert torch.equal(mine, out.view)
        dy, dw, db = E.mix_backward(dout, yy, index, w, experts)
        ody, odw = Out(tokens * k, cols, dtype, pad, lead), Out(tokens, k, F32)
        args = (put(dout, pad, lead), put(yy, pad, lead), index.cuda(), None if w is None else w.cuda())
        zo.zero_expert_mix_backward(*args, ody.view, odw.view, experts=experts)
        torch.cuda.synchronize()
        assert ody.guards_intact() and odw.guards_intact()
        C.within(ody.view, dy, C.rounded(C.U * dy.abs(), dy, dtype), "dy")
        C.within(odw.view, dw, db, "dweight")
        mine = put(yy, pad, lead)
        zo.zero_expert_mix_backward(args[0], mine, *args[2:], mine, odw.view, experts=experts)
        assert torch.equal(mine, ody.view)
        only = torch.empty(tokens * k, cols, dtype=dtype, device="cuda")  # each output alone
        zo.zero_expert_mix_backward(args[0], None, *args[2:], only, experts=experts)
        assert torch.equal(only, ody.view)
        alone = torch.empty(tokens, k, device="cuda")
        zo.zero_expert_mix_backward(*args, None, alone, experts=experts)
        assert torch.equal(alone, odw.view)


def test_mix_without_tokens(zo):
    none = torch.empty(0, 16, dtype=F16, device="cuda")
    index = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    zo.zero_expert_mix(none, index, none.clone())
    zo.zero_expert_mix_backward(none, none.clone(), index, None, none.clone(), torch.empty(0, 3, device="cuda"))


def layer(zo, x, router, up, down, k, room, order_room, bufs):
    """The experts' layer as a training program calls it: route, order, two products with a ReLU, mixing; then the
    gradients of everything from dout."""
    tokens, hidden = x.shape
    experts, inner = up.shape[0], up.shape[2]
    b = bufs
    zo.zero_route(b["logits"], b["index"], b["weight"])
    zo.zero_route_order(b["index"], experts, b["offsets"], b["order"], order_room)
    zo.zero_expert_product(x, up, b["offsets"], b["inner"], order=b["order"], x_slots=k)
    b["inner"].clamp_(min=0)
    zo.zero_expert_product(b["inner"], down, b["offsets"], b["y"], order=b["order"], y_slots=1)
    zo.zero_expert_mix(b["y"], b["index"], b["out"], weight=b["weight"], base=x)
    zo.zero_expert_mix_backward(b["dout"], b["y"], b["index"], b["weight"], b["dy"], b["dweight"])
    zo.zero_expert_weight_backward(b["inner"], b["dy"], b["offsets"], b["ddown"], room, order=b["order"], dy_slots=1)
    zo.zero_expert_product(b["dy"], down, b["offsets"], b["dinner"], order=b["order"], x_slots=1, transposed=True)
    b["dinner"].mul_(b["inner"] > 0)
    zo.zero_expert_weight_backward(x, b["dinner"], b["offsets"], b["dup"], room, order=b["order"], x_slots=k)
    zo.zero_expert_product(b["dinner"], up, b["offsets"], b["dslots"], order=b["order"], y_slots=1, transposed=True)
    zo.zero_expert_mix(b["dslots"], b["index"], b["dx"], base=b["dout"])
    zo.zero_route_backward(b["logits"], b["index"], b["dweight"], b["dlogits"])


def layer_buffers(tokens, hidden, inner, experts, k, dtype, seed):
    g = C.rng(seed, tokens)
    x, dout = C.normal(g, tokens, hidden).to(dtype), C.normal(g, tokens, hidden).to(dtype)
    logits = C.normal(g, tokens, experts).to(dtype)
    up = (C.normal(g, experts, hidden, inner) * hidden ** -0.5).to(dtype)
    down = (C.normal(g, experts, inner, hidden) * inner ** -0.5).to(dtype)
    new = lambda *s, t=dtype: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    n = tokens * k
    bufs = dict(logits=logits.cuda(), dout=dout.cuda(), index=new(tokens, k, t=torch.int32), weight=new(tokens, k, t=F32),
                offsets=new(experts + 1, t=torch.int32), order=new(n, t=torch.int32), inner=new(n, inner), y=new(n, hidden),
                out=new(tokens, hidden), dy=new(n, hidden), dweight=new(tokens, k, t=F32), ddown=new(experts, inner, hidden),
                dinner=new(n, inner), dup=new(experts, hidden, inner), dslots=new(n, hidden), dx=new(tokens, hidden),
                dlogits=new(tokens, experts))
    return x, logits, up, down, dout, bufs


def test_layer_against_autograd(zo):
    """In fp32: every gradient of the layer against float64 automatic differentiation.  Sums of up to 600 terms of
    order 1 in two products one after another: 1e-5 of the largest element is 80 units."""
    tokens, hidden, inner, experts, k = 150, 40, 72, 5, 2
    x, logits, up, down, dout, b = layer_buffers(tokens, hidden, inner, experts, k, F32, 31)
    n = max(zo.zero_expert_workspace(tokens * k, experts, hidden, inner),
            zo.zero_expert_workspace(tokens * k, experts, inner, hidden), 1)
    layer(zo, x.cuda(), None, up.cuda(), down.cuda(), k, torch.empty(n, device="cuda"), None, b)
    xd, zd, ud, dd = (t.double().requires_grad_(True) for t in (x, logits, up, down))
    index = b["index"].cpu().long()
    w = torch.softmax(zd.gather(1, index), 1)
    out = xd.clone()
    for i in range(k):
        h = torch.relu(torch.einsum("th,thj->tj", xd, ud[index[:, i]]))
        out = out + w[:, i, None] * torch.einsum("tj,tjh->th", h, dd[index[:, i]])
    grads = torch.autograd.grad((out * dout.double()).sum(), (xd, zd, ud, dd))
    for name, want in (("out", out.detach()), ("dx", grads[0]), ("dlogits", grads[1]), ("dup", grads[2]),
                       ("ddown", grads[3])):
        err = (b[name].cpu().double() - want).abs().max() / want.abs().max()
        assert err < 1e-5, (name, err)


def test_gradients_against_differences(zo):
    """d sum(y dy) / d weight and / d x by central differences of the fp32 product, which is linear in each: the
    rounding of sums of 40 terms of order 1 over the step, 2^-24 * 40 * 200 / 2^-3, stays under 4e-3."""
    index, offsets, placed = E.choice(6, 2, 3, 41)
    g = C.rng(43)
    x, w, dy = C.normal(g, 6, 10).float(), C.normal(g, 3, 10, 9).float(), C.normal(g, 12, 9).float()
    o, p = offsets.cuda(), placed.cuda()

    def loss(x, w):
        y = torch.zeros(12, 9, device="cuda")
        zo.zero_expert_product(x.cuda(), w.cuda(), o, y, order=p, x_slots=2, y_slots=1)
        return float((y.cpu().double() * dy.double()).sum())

    dw, dslots, dx = torch.empty(3, 10, 9, device="cuda"), torch.zeros(12, 10, device="cuda"), torch.empty(6, 10, device="cuda")
    zo.zero_expert_weight_backward(x.cuda(), dy.cuda(), o, dw, order=p, x_slots=2, dy_slots=1)
    zo.zero_expert_product(dy.cuda(), w.cuda(), o, dslots, order=p, x_slots=1, y_slots=1, transposed=True)
    zo.zero_expert_mix(dslots, index.cuda(), dx)
    step = 2.0 ** -3
    for at in ((0, 3, 2), (1, 9, 8), (2, 0, 0)):
        d = torch.zeros_like(w)
        d[at] = step
        assert abs((loss(x, w + d) - loss(x, w - d)) / (2 * step) - dw[at].item()) < 4e-3
    for at in ((0, 0), (5, 9), (3, 4)):
        d = torch.zeros_like(x)
        d[at] = step
        assert abs((loss(x + d, w) - loss(x - d, w)) / (2 * step) - dx[at].item()) < 4e-3


def test_layer_in_a_graph_and_on_a_stream(zo):
    """Captured once, replayed on new inputs between eager calls, on a stream of its own; the same bits every time."""
    tokens, hidden, inner, experts, k = 1500, 64, 96, 4, 2
    x, _, up, down, _, b = layer_buffers(tokens, hidden, inner, experts, k, F16, 33)
    x, up, down = x.cuda(), up.cuda(), down.cuda()
    n = max(zo.zero_expert_workspace(tokens * k, experts, hidden, inner),
            zo.zero_expert_workspace(tokens * k, experts, inner, hidden))
    assert n > 0
    room = torch.empty(n, device="cuda")
    order_room = torch.empty(max(1, zo.zero_route_workspace(tokens * k, experts)), dtype=torch.int32, device="cuda")

    def go():
        layer(zo, x, None, up, down, k, room, order_room, b)

    names = ("out", "dx", "dlogits", "dup", "ddown", "dweight")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        go()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            go()
        for turn in range(4):
            x.mul_(0.75)
            b["logits"].neg_()
            go()
            want = {m: b[m].clone() for m in names}
            for m in names:
                b[m].zero_()
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(b[m], want[m]) for m in names), turn


def test_offsets_past_32_bits(zo):
    """Rows far apart: the last row of each matrix lies past 2^32 elements from the first."""
    ld, rows = (1 << 31) + 64, 3
    buf = torch.zeros((rows - 1) * ld + 1024, dtype=F16, device="cuda")
    x = torch.as_strided(buf, (rows, 64), (ld, 1))
    x.copy_(torch.randn(rows, 64, device="cuda"))
    y, out = (torch.as_strided(buf, (rows, 64), (ld, 1), 128 * (i + 1)) for i in range(2))
    w = (torch.randn(1, 64, 64, device="cuda") / 8).half()
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    order = torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda")
    far = torch.as_strided(buf, (1, 2, 64), (0, ld, 1), 512)   # weights whose rows lie far apart
    far.copy_(w[:, :2])
    for layout in (0, 1):
        zo.zero_expert_product(x, w, offsets, y, order=order, x_slots=layout, y_slots=1)
        rr = torch.arange(3, device="cuda") if layout == 0 else order.long()
        want = torch.empty(rows, 64, device="cuda")
        want[order.long()] = x[rr].float() @ w[0].float()
        assert (y.float() - want).abs().max() < 2e-2  # of values up to 4 or so: 2^-11 of them and 64 sums
    two = torch.empty(rows, 64, dtype=F16, device="cuda")
    x2 = x[:, :2].contiguous()
    zo.zero_expert_product(x2, far, offsets, two)
    assert (two.float() - x2.float() @ far[0].float()).abs().max() < 1e-2
    dw = torch.empty(1, 64, 64, dtype=F16, device="cuda")
    zo.zero_expert_weight_backward(x, y, offsets, dw, order=order, x_slots=1, dy_slots=1)
    want = x.float().t() @ y.float()
    assert (dw[0].float() - want).abs().max() < 2e-2 * want.abs().max()
    index = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    zo.zero_expert_mix(y, index, out, base=x)
    assert (out.float() - (y.float() + x.float())).abs().max() < 1e-2
    d = torch.empty(rows, 1, device="cuda")
    zo.zero_expert_mix_backward(x, y, index, None, out, d)
    assert torch.equal(out, x) and (d[:, 0] - (x.float() * y.float()).sum(1)).abs().max() < 1e-2
