"""The experts' products and their weights' gradient on each way of their operands to LDS, chosen by size and
alignment: through registers, and as aligned chunks; against the plain 64-bit implementations of expert_checks.py."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import expert_checks as E  # noqa: E402
import operator_checks as C  # noqa: E402
from test_gpu_expert_runs import weights  # noqa: E402
from test_gpu_experts import run_product, zo  # noqa: E402,F401
from test_gpu_operators import Out, put  # noqa: E402

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


# Through registers the copies are a step further ahead of the products than they are straight to LDS: with tiles
# of one step (64 columns of 16 bits) the third tile's rows are looked up before the first has ended.
@pytest.mark.parametrize("dtype", (F16, BF16))
@pytest.mark.parametrize("x_slots,y_slots", ((1, 0), (2, 1)))
@pytest.mark.parametrize("slots,experts,cin,cout,lead", (
    (1700, 12, 50, 10001, 1), (2600, 3, 64, 10000, 1), (2600, 3, 1, 10000, 0), (6000, 100, 63, 2600, 1)))
def test_product_tiles_of_one_step_through_registers(zo, slots, experts, cin, cout, lead, x_slots, y_slots, dtype):  # noqa: F811
    for transposed in (False, True):
        run_product(zo, slots // 2, 2, experts, cin, cout, dtype, x_slots, y_slots, transposed, 0, lead, 0.02)


# An output or operand of Out and put begins 37 elements from an aligned address, so `lead` 3 makes its rows aligned
# chunks of 16 bytes where their width and distance allow it; those go straight to LDS.
LEAD = 3


def test_the_lead_that_aligns(zo):  # noqa: F811
    for dtype in C.TYPES:
        assert put(torch.zeros(2, 8, dtype=dtype), 8, LEAD).data_ptr() % 16 == 0
        assert put(torch.zeros(2, 8, dtype=dtype), 8, 1).data_ptr() % 16 != 0


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,experts,cin,cout,pad", (
    (1, 1, 1, 8, 8, 0), (1, 2, 4, 8, 8, 8), (3, 2, 5, 16, 24, 0), (8, 6, 64, 128, 136, 0), (37, 3, 7, 200, 24, 8),
    (1, 1, 1024, 64, 32, 0), (40, 2, 3, 72, 136, 0), (32, 1, 1, 256, 128, 0), (33, 1, 1, 320, 264, 0),
    (48, 2, 2, 520, 264, 0), (300, 2, 16, 584, 392, 8)))
def test_product_of_few_rows_straight_to_lds(zo, tokens, k, experts, cin, cout, pad, dtype):  # noqa: F811
    for transposed in (False, True):
        run_product(zo, tokens, k, experts, cin, cout, dtype, 0, 0, transposed, pad, LEAD)
        run_product(zo, tokens, k, experts, cin, cout, dtype, k, 1, transposed, pad, LEAD, 0.1)
        run_product(zo, tokens, k, experts, cin, cout, dtype, 1, 0, transposed, pad, LEAD, 0.1)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,experts,cin,cout,pad", (
    (130, 2, 2, 264, 264, 0), (257, 2, 1, 96, 136, 8), (300, 4, 2, 72, 264, 0), (700, 2, 2, 136, 304, 0),
    (500, 1, 3, 8, 8, 0), (400, 2, 3, 1032, 520, 8)))
def test_product_straight_to_lds(zo, tokens, k, experts, cin, cout, pad, dtype):  # noqa: F811
    for transposed in (False, True):
        for x_slots, y_slots in ((0, 0), (1, 0), (k, 1), (0, 1)):
            run_product(zo, tokens, k, experts, cin, cout, dtype, x_slots, y_slots, transposed, pad, LEAD, 0.05)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("rows", (127, 128, 129, 255, 256, 257, 511, 513))
def test_product_rows_about_a_tile_straight_to_lds(zo, rows, dtype):  # noqa: F811
    for transposed in (False, True):
        run_product(zo, rows, 1, 1, 136, 264, dtype, 1, 1, transposed, 0, LEAD)


# several tiles for each workgroup, of 256 rows (2600 and 5200 slots) or 128, of one step, two, three, four and seven
@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("transposed", (False, True))
@pytest.mark.parametrize("slots,experts,cin,cout,pad", (
    (2600, 3, 64, 10000, 0), (2600, 3, 72, 10000, 8), (2600, 3, 200, 10008, 0), (5200, 2, 136, 5200, 0),
    (1700, 12, 24, 10000, 0), (1700, 12, 128, 10000, 0), (1700, 12, 440, 8200, 0)))
def test_product_many_tiles_a_workgroup_straight_to_lds(zo, slots, experts, cin, cout, pad, transposed, dtype):  # noqa: F811
    cout = cout if dtype != F32 else cout // 2
    run_product(zo, slots // 2, 2, experts, cin, cout, dtype, 2, 1, transposed, pad, LEAD, 0.05)
    if transposed:
        run_product(zo, slots // 2, 2, experts, cin, cout, dtype, 1, 0, transposed, pad, LEAD)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,experts,cin,cout,pad", (
    (1, 1, 1, 8, 8, 0), (3, 2, 5, 8, 16, 8), (8, 6, 64, 16, 24, 0), (130, 2, 2, 136, 264, 0), (2100, 2, 2, 24, 40, 0),
    (1, 1, 1024, 8, 8, 0), (100, 2, 40, 1000, 1304, 0), (20, 1, 300, 264, 520, 0),
    (63, 1, 1, 264, 136, 0), (64, 1, 1, 264, 264, 0), (65, 1, 1, 264, 264, 0)))
def test_weight_backward_straight_to_lds(zo, tokens, k, experts, cin, cout, pad, dtype):  # noqa: F811
    weights(zo, tokens, k, experts, cin, cout, dtype, k, 1, pad, LEAD, 0.05)
    weights(zo, tokens, k, experts, cin, cout, dtype, 0, 0, pad, LEAD)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("only", ([2], [0, 4], [4]))
@pytest.mark.parametrize("cin,cout,pad", ((96, 200, 0), (264, 304, 8)))
def test_weight_backward_of_one_long_expert_straight_to_lds(zo, cin, cout, pad, only, dtype):  # noqa: F811
    assert zo.zero_expert_workspace(6000, 5, cin, cout) > 0
    weights(zo, 3000, 2, 5, cin, cout, dtype, 2, 1, pad, LEAD, 0.01, only)
    weights(zo, 3000, 2, 5, cin, cout, dtype, 0, 0, pad, LEAD, 0.0, only)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("lead", (0, LEAD))
@pytest.mark.parametrize("tokens,cin,cout", ((600, 40, 264), (600, 200, 264), (90, 200, 264), (20, 40, 136)))
def test_entries_of_order_that_name_no_slot(zo, tokens, cin, cout, lead, dtype):  # noqa: F811
    """They give rows of zeros where x is read, none where y is written, nothing to the weights' gradient; the row of x
    that is read in their place (the first, which no slot here takes) may hold NaN.  300, 45 and 10 rows an expert."""
    k, experts = 2, 4
    slots = tokens * k
    g = C.rng(41, tokens, cin)
    index = torch.randint(0, experts, (tokens, k), generator=g)
    index[0] = -1
    offsets, placed = (torch.tensor(t, dtype=torch.int32) for t in C.order(index, experts))
    bad = placed.clone()
    n = int(offsets[-1])
    hit = sorted({5 * n // 37, 13 * n // 37, 22 * n // 37, n - 1, 0})
    bad[hit] = torch.tensor([-1, slots, 2 ** 31 - 1, -2 ** 31, slots + 7], dtype=torch.int32)[:len(hit)]
    x, w = C.normal(g, tokens, cin).to(dtype), C.normal(g, experts, cin, cout).to(dtype)
    x[0] = math.nan
    dx, o, b = put(x, 0, lead), offsets.cuda(), bad.cuda()
    clean = torch.where(torch.isnan(x), 0, x)
    for transposed in (False, True):
        ww = w.transpose(1, 2).contiguous() if transposed else w
        dw = put(ww.flatten(0, 1), 0, lead).unflatten(0, (experts, -1))
        want, bound, written = E.product(clean, ww, offsets, placed, k, 0, transposed, slots)
        want[hit], bound[hit] = 0, 0
        out = Out(slots, cout, dtype, 0, lead)
        zo.zero_expert_product(dx, dw, o, out.view, order=b, x_slots=k, transposed=transposed)
        torch.cuda.synchronize()
        assert out.guards_intact()
        assert (out.view.cpu()[~written].view(-1).view(torch.uint8) == 0xA5).all()
        C.within(out.view.cpu()[written], want[written], C.rounded(bound, want, dtype)[written], "y")
        assert (out.view[hit] == 0).all()
        # in the slots' order, from rows of either order
        xs = clean[placed[:n].long() // k]
        for x_slots, from_ in ((k, dx), (0, put(torch.cat([xs, torch.zeros(slots - n, cin).to(dtype)]), 0, lead))):
            want, bound, written = E.product(clean, ww, offsets, placed, k, 1, transposed, slots)
            written[placed[hit].long()] = False
            out = Out(slots, cout, dtype, 0, lead)
            zo.zero_expert_product(from_, dw, o, out.view, order=b, x_slots=x_slots, y_slots=1, transposed=transposed)
            torch.cuda.synchronize()
            assert out.guards_intact()
            assert (out.view.cpu()[~written].view(-1).view(torch.uint8) == 0xA5).all()
            C.within(out.view.cpu()[written], want[written], C.rounded(bound, want, dtype)[written], "y by slot")
    dy = C.normal(g, slots, cout).to(dtype)
    for dy_slots in (0, 1):
        gone = dy.clone()
        gone[placed[hit].long() if dy_slots else hit] = 0
        want, bound = E.weight_backward(clean, gone, offsets, placed, k, dy_slots)
        bound = bound + 64 * C.U * want.abs()  # of sums in parts
        room = Out(1, zo.zero_expert_workspace(slots, experts, cin, cout), F32)
        out = Out(experts * cin, cout, dtype, 0, lead)
        zo.zero_expert_weight_backward(dx, put(dy, 0, lead), o, out.view.unflatten(0, (experts, cin)), room.view[0], order=b,
                                       x_slots=k, dy_slots=dy_slots)
        torch.cuda.synchronize()
        assert out.guards_intact() and room.guards_intact()
        C.within(out.view.unflatten(0, (experts, cin)), want, C.rounded(bound, want, dtype), "dw")


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,cols", ((1, 1, 5), (7, 3, 264), (40, 8, 130)))
def test_mix_where_every_slot_has_an_expert(zo, tokens, k, cols, dtype):  # noqa: F811
    """Without an index k is that of y's rows, and nothing is left out."""
    g = C.rng(43, tokens, k, cols)
    y, dout, w = C.normal(g, tokens * k, cols).to(dtype), C.normal(g, tokens, cols).to(dtype), C.normal(g, tokens, k).float()
    every = torch.zeros(tokens, k, dtype=torch.int32)
    dy, dw, db = E.mix_backward(dout, y, every, w)
    yd, dd = y.cuda(), dout.cuda()
    for weight in (None, w):
        want, bound = E.mix(y, every, weight, None)
        out = torch.empty_like(dd)
        zo.zero_expert_mix(yd, None, out, weight=None if weight is None else weight.cuda())
        C.within(out, want, C.rounded(bound, want, dtype), "out")
    got, gw = torch.empty_like(yd), torch.empty(tokens, k, device="cuda")
    zo.zero_expert_mix_backward(dd, yd, None, w.cuda(), got, gw)
    C.within(got, dy, C.rounded(C.U * dy.abs(), dy, dtype), "dy")
    C.within(gw, dw, db, "dweight")
    alone = torch.empty_like(yd)
    zo.zero_expert_mix_backward(dd, None, None, w.cuda(), alone)
    assert torch.equal(alone, got)
    none = torch.empty(0, cols, dtype=dtype, device="cuda")
    zo.zero_expert_mix(none, None, none.clone())
    with pytest.raises(ValueError):
        zo.zero_expert_mix(yd, None, torch.empty(tokens + 1, cols, dtype=dtype, device="cuda"))
    with pytest.raises(ValueError):
        zo.zero_expert_mix_backward(dd, None, None, w.cuda(), None)


@pytest.mark.parametrize("lead", (0, LEAD))
@pytest.mark.parametrize("rows,cin,cout", ((20, 262144, 8), (60, 262144, 8), (20, 8193, 40), (60, 5000, 72), (130, 65536, 16)))
def test_long_sums_in_fp32(zo, rows, cin, cout, lead):  # noqa: F811
    """512 products in a chain, then a rounding for each 512: the bound does not grow with the length.  Equal products,
    whose roundings in one chain all go the same way, and numbers of either sign."""
    g = C.rng(47, rows, cin)
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    for x, w in ((torch.full((rows, cin), 0.9), torch.ones(cin, cout)),
                 (C.normal(g, rows, cin).float(), C.normal(g, cin, cout).float())):
        want, size = x.double() @ w.double(), x.double().abs() @ w.double().abs()
        bound = (512 + cin / 512 + 8) * 2 * C.U * size
        for transposed in (False, True):
            ww = w.t().contiguous() if transposed else w
            out = Out(rows, cout, F32, 0, lead)
            zo.zero_expert_product(put(x, 0, lead), put(ww, 0, lead).unsqueeze(0), offsets, out.view, transposed=transposed)
            torch.cuda.synchronize()
            assert out.guards_intact()
            C.within(out.view, want, C.rounded(bound, want, F32), "y")


@pytest.mark.parametrize("lead", (0, 1))
@pytest.mark.parametrize("rows,cin,cout,parts", ((8193, 2900, 2904, False), (40000, 4100, 4100, False), (100000, 40, 72, True)))
def test_long_sums_of_the_weights_gradient_in_fp32(zo, rows, cin, cout, parts, lead):  # noqa: F811
    """As above, over an expert's rows: in one part, or in several whose sums are added up."""
    n = zo.zero_expert_workspace(rows, 1, cin, cout)
    assert (n > 0) == parts

    def full(cols, value):
        return torch.full((lead + rows * cols,), value, device="cuda")[lead:].view(rows, cols)

    out = Out(cin, cout, F32, 0, lead)
    room = Out(1, n, F32)
    zo.zero_expert_weight_backward(full(cin, 0.9), full(cout, 1.0), torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                                   out.view.unsqueeze(0), room.view[0])
    torch.cuda.synchronize()
    assert out.guards_intact() and room.guards_intact()
    want = rows * torch.tensor(0.9).double().item()
    assert (out.view.double() - want).abs().max().item() <= (512 + rows / 512 + 8) * 2 * C.U * want
