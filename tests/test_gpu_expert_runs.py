"""The experts' products and their weights' gradient where a workgroup takes many tiles one after another, where tiles have
few steps or none, where one expert has nearly all rows, and beside each other on two streams; against the plain 64-bit
implementations of expert_checks.py."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import expert_checks as E  # noqa: E402
import operator_checks as C  # noqa: E402
from test_gpu_experts import run_product, zo  # noqa: E402,F401
from test_gpu_operators import Out, put  # noqa: E402

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


# 256 compute units take tiles of 256 or 128 rows by 256 columns (fp32: 64 by 64): several tiles for each workgroup, of
# one step, of two, the last of them short, and of seven
@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("transposed", (False, True))
@pytest.mark.parametrize("slots,experts,cin,cout,pad,lead", (
    (2600, 3, 64, 17000, 0, 0), (2600, 3, 72, 17000, 8, 0), (1700, 12, 24, 17000, 0, 0), (1700, 12, 440, 8200, 0, 0),
    (1700, 12, 65, 17001, 0, 1)))
def test_product_many_tiles_a_workgroup(zo, slots, experts, cin, cout, pad, lead, transposed, dtype):  # noqa: F811
    cout = cout if dtype != F32 else cout // 2
    run_product(zo, slots // 2, 2, experts, cin, cout, dtype, 2, 1, transposed, pad, lead, 0.05)
    run_product(zo, slots // 2, 2, experts, cin, cout, dtype, 0, 0, transposed, pad, lead)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("lead", (0, 1))
@pytest.mark.parametrize("rows", (1, 127, 128, 129, 255, 256, 257, 511, 513))
def test_product_rows_about_a_tile(zo, rows, lead, dtype):  # noqa: F811
    for transposed in (False, True):
        run_product(zo, rows, 1, 1, 136, 264, dtype, 1, 1, transposed, 0, lead)


def weights(zo, tokens, k, experts, cin, cout, dtype, x_slots, dy_slots, pad=0, lead=0, none=0.0, only=None):  # noqa: F811
    _, offsets, placed = E.choice(tokens, k, experts, 3, none, only)
    slots = tokens * k
    g = C.rng(7, cin, cout)
    x = C.normal(g, slots // x_slots if x_slots > 1 else slots, cin).to(dtype)
    dy = C.normal(g, slots // dy_slots if dy_slots > 1 else slots, cout).to(dtype)
    want, bound = E.weight_backward(x, dy, offsets, placed, x_slots, dy_slots)
    # what is summed in parts is rounded once a part more, to fp32, and the parts are added up
    bound = bound + 64 * C.U * want.abs()
    out = Out(experts * cin, cout, dtype, pad, lead)
    room = Out(1, zo.zero_expert_workspace(slots, experts, cin, cout), F32)
    args = (put(x, pad, lead), put(dy, pad, lead), offsets.cuda())
    kw = dict(order=placed.cuda() if x_slots or dy_slots else None, x_slots=x_slots, dy_slots=dy_slots)
    zo.zero_expert_weight_backward(*args, out.view.unflatten(0, (experts, cin)), room.view[0], **kw)
    torch.cuda.synchronize()
    assert out.guards_intact() and room.guards_intact()
    C.within(out.view.unflatten(0, (experts, cin)), want, C.rounded(bound, want, dtype), "dw")
    again = torch.empty(experts, cin, cout, dtype=dtype, device="cuda")
    zo.zero_expert_weight_backward(*args, again, room.view[0], **kw)
    assert torch.equal(again.view(-1, cout), out.view)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("tokens,k,experts,cin,cout,pad,lead", (
    (200, 2, 40, 1000, 1304, 0, 0),   # 20 to 48 tiles of 40 experts of 10 rows
    (700, 3, 24, 520, 2056, 8, 0), (300, 2, 30, 1001, 777, 0, 1), (20, 1, 300, 264, 520, 0, 0)))
def test_weight_backward_many_tiles_a_workgroup(zo, tokens, k, experts, cin, cout, pad, lead, dtype):  # noqa: F811
    weights(zo, tokens, k, experts, cin, cout, dtype, k, 1, pad, lead, 0.05)


@pytest.mark.parametrize("dtype", C.TYPES)
@pytest.mark.parametrize("only", ([2], [0, 4], [4]))
@pytest.mark.parametrize("cin,cout,pad,lead", ((96, 200, 0, 0), (264, 304, 8, 0), (67, 129, 0, 1)))
def test_weight_backward_of_one_long_expert(zo, cin, cout, pad, lead, only, dtype):  # noqa: F811
    """Parts of one expert's rows, beside experts without rows."""
    assert zo.zero_expert_workspace(6000, 5, cin, cout) > 0
    weights(zo, 3000, 2, 5, cin, cout, dtype, 2, 1, pad, lead, 0.01, only)
    weights(zo, 3000, 2, 5, cin, cout, dtype, 0, 0, pad, lead, 0.0, only)


@pytest.mark.parametrize("rows", (255, 256, 257, 511, 512, 513, 64, 63, 65, 1))
def test_weight_backward_rows_about_a_part(zo, rows):  # noqa: F811
    weights(zo, rows, 1, 1, 72, 136, BF16, 1, 1)


def test_offsets_that_fall(zo):  # noqa: F811
    """An offset below one before it counts as that one: the rows of every expert are its own, in parts too."""
    tokens, cin, cout = 3000, 64, 72
    offsets = torch.tensor([0, 1500, 700, 1600, 100, 3000], dtype=torch.int32)
    clean = torch.cummax(offsets, 0).values.int()
    g = C.rng(5)
    x, dy = C.normal(g, tokens, cin).to(BF16), C.normal(g, tokens, cout).to(BF16)
    w = C.normal(g, 5, cin, cout).to(BF16)
    placed = torch.arange(tokens).int()
    want, bound, _ = E.product(x, w, clean, placed, 0, 0, False, tokens)
    y = torch.empty(tokens, cout, dtype=BF16, device="cuda")
    zo.zero_expert_product(x.cuda(), w.cuda(), offsets.cuda(), y)
    C.within(y, want, C.rounded(bound, want, BF16), "y")
    want, bound = E.weight_backward(x, dy, clean, placed, 0, 0)
    room = torch.empty(zo.zero_expert_workspace(tokens, 5, cin, cout), device="cuda")
    assert room.numel() > 0
    dw = torch.empty(5, cin, cout, dtype=BF16, device="cuda")
    zo.zero_expert_weight_backward(x.cuda(), dy.cuda(), offsets.cuda(), dw, room)
    C.within(dw, want, C.rounded(bound + 64 * C.U * want.abs(), want, BF16), "dw")


def test_two_streams_at_once(zo):  # noqa: F811
    """Calls beside each other, each with buffers and workspace of its own, have the bits that they have alone."""
    tokens, k, experts, cin, cout = 2000, 2, 6, 136, 264
    _, offsets, placed = E.choice(tokens, k, experts, 9)
    o, p = offsets.cuda(), placed.cuda()
    n = zo.zero_expert_workspace(tokens * k, experts, cin, cout)
    calls = []
    for seed in (1, 2):
        g = C.rng(seed)
        x, dy = C.normal(g, tokens, cin).to(F16).cuda(), C.normal(g, tokens * k, cout).to(F16).cuda()
        w = C.normal(g, experts, cin, cout).to(F16).cuda()
        y, dw = torch.zeros(tokens * k, cout, dtype=F16, device="cuda"), torch.zeros(experts, cin, cout, dtype=F16, device="cuda")
        calls.append((x, dy, w, y, dw, torch.empty(n, device="cuda")))

    def go(x, dy, w, y, dw, room, stream):
        zo.zero_expert_product(x, w, o, y, order=p, x_slots=k, y_slots=1, stream=stream)
        zo.zero_expert_weight_backward(x, dy, o, dw, room, order=p, x_slots=k, dy_slots=1, stream=stream)

    alone = []
    for c in calls:
        go(*c, None)
        torch.cuda.synchronize()
        alone.append((c[3].clone(), c[4].clone()))
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for c in calls:
            c[3].zero_()
            c[4].zero_()
        torch.cuda.synchronize()
        for c, s in zip(calls, streams):
            go(*c, s)
        torch.cuda.synchronize()
        for c, (y, dw) in zip(calls, alone):
            assert torch.equal(c[3], y) and torch.equal(c[4], dw)
