"""The C ABI and binding of the experts' operators and of zero_log_probs without a GPU: records laid out alike in C and
Python, wrong arguments refused before any HIP call, and the checks that the GPU tests use against automatic
differentiation and planted mistakes."""
import math
import os
import shutil
import subprocess
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import expert_checks as E  # noqa: E402
import log_prob_checks as L  # noqa: E402
import operator_checks as C  # noqa: E402
from test_operators_cpu import ROOT, fields, zo  # noqa: E402,F401

RECORDS = {"zero_expert_product_args_t": "EXPERT_PRODUCT_ARGS",
           "zero_expert_weight_backward_args_t": "EXPERT_WEIGHT_BACKWARD_ARGS",
           "zero_expert_mix_args_t": "EXPERT_MIX_ARGS", "zero_expert_mix_backward_args_t": "EXPERT_MIX_BACKWARD_ARGS",
           "zero_log_probs_args_t": "LOG_PROBS_ARGS", "zero_log_probs_backward_args_t": "LOG_PROBS_BACKWARD_ARGS"}


@pytest.mark.parametrize("record", sorted(RECORDS))
def test_records_have_the_headers_fields(zo, record):  # noqa: F811
    code = {"int32_t": "i", "int64_t": "q", "double": "d"}
    want = "".join("P" if t.endswith("*") else code[t] for t, _ in fields(record))
    assert getattr(zo, RECORDS[record]).format == "@" + want


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_records_have_the_compilers_sizes(zo, tmp_path):  # noqa: F811
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text('#include <stdio.h>\n#include "zero_operators.h"\nint main(void) {\n' + "".join(
        'printf("%s %%zu\\n", sizeof(%s));\n' % (r, r) for r in RECORDS) + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe)], check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], stdout=subprocess.PIPE, check=True).stdout.decode()
               .splitlines())
    assert {r: int(n) for r, n in got.items()} == {r: getattr(zo, p).size for r, p in RECORDS.items()}


# Addresses that no call may get to dereference or look up: every call below is refused before.
A = [0x10000000 * (i + 1) for i in range(12)]
GOOD = {
    "zero_expert_product": ("zero_expert_product_args_t", dict(
        dtype=1, experts=4, slots=24, cols_in=64, cols_out=32, transposed=0, x_slots=2, y_slots=1, pad_=0, offsets=A[0],
        order=A[1], x=A[2], ld_x=64, weight=A[3], ld_weight=32, y=A[4], ld_y=32)),
    "zero_expert_weight_backward": ("zero_expert_weight_backward_args_t", dict(
        dtype=1, experts=2, slots=4096, cols_in=64, cols_out=32, x_slots=2, dy_slots=1, offsets=A[0], order=A[1], x=A[2],
        ld_x=64, dy=A[3], ld_dy=32, dweight=A[4], ld_dweight=32, workspace=A[5], workspace_floats=1 << 24)),
    "zero_expert_mix": ("zero_expert_mix_args_t", dict(
        dtype=2, k=2, tokens=5, cols=64, experts=8, pad_=0, index=A[0], weight=A[1], y=A[2], ld_y=64, base=A[3], ld_base=64,
        out=A[4], ld_out=64)),
    "zero_expert_mix_backward": ("zero_expert_mix_backward_args_t", dict(
        dtype=2, k=2, tokens=5, cols=64, experts=8, pad_=0, index=A[0], weight=A[1], dout=A[2], ld_dout=64, y=A[3], ld_y=64,
        dy=A[4], ld_dy=64, dweight=A[5])),
    "zero_log_probs": ("zero_log_probs_args_t", dict(
        dtype=0, k=5, rows=4, vocab=1000, temperature=1.0, logits=A[0], ld_logits=1000, tokens=A[1], logp=A[2], entropy=A[3],
        top_index=A[4], top_logp=A[5], stats=A[6])),
    "zero_log_probs_backward": ("zero_log_probs_backward_args_t", dict(
        dtype=0, pad_=0, rows=4, vocab=1000, temperature=1.0, grad_scale=64.0, logits=A[0], ld_logits=1000, tokens=A[1],
        stats=A[2], dlogp=A[3], dentropy=A[4], dlogits=A[5], ld_dlogits=1000)),
}
NAN, INF = math.nan, math.inf
SIZES = (dict(dtype=3), dict(dtype=-1), dict(experts=0), dict(experts=1025), dict(slots=-1), dict(slots=1 << 31),
         dict(cols_in=0), dict(cols_in=(1 << 20) + 1), dict(cols_out=0), dict(cols_out=1 << 21), dict(x_slots=-1),
         dict(x_slots=5), dict(x_slots=7), dict(order=0), dict(offsets=0), dict(x=0), dict(ld_x=63), dict(x=A[2] + 1),
         dict(order=A[1] + 2), dict(offsets=A[0] + 1), dict(ld_x=1 << 41))
MIX = (dict(dtype=5), dict(k=0), dict(k=65), dict(tokens=-1), dict(tokens=1 << 30), dict(cols=0), dict(cols=(1 << 20) + 1),
       dict(experts=-1), dict(index=A[0] + 2), dict(weight=A[1] + 1), dict(ld_y=63), dict(y=A[3] + 1))
ROWS = (dict(dtype=9), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(temperature=0.0), dict(temperature=-1.0),
        dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-31), dict(temperature=1e31), dict(logits=0),
        dict(ld_logits=999), dict(logits=A[0] + 2), dict(tokens=0))
BAD = [("zero_expert_product", c) for c in SIZES + (
    dict(y_slots=2), dict(y_slots=-1), dict(weight=0), dict(y=0), dict(ld_weight=31), dict(transposed=1), dict(ld_y=10),
    dict(y=A[2]), dict(y=A[3] + 64), dict(y=A[1]))
] + [("zero_expert_weight_backward", c) for c in SIZES + (
    dict(dy_slots=3), dict(dy_slots=-2), dict(dy=0), dict(dweight=0), dict(ld_dy=31), dict(ld_dweight=4), dict(dweight=A[2]),
    dict(dweight=A[3]), dict(workspace=0), dict(workspace=A[4]), dict(workspace_floats=100), dict(workspace_floats=-1),
    dict(workspace=A[5] + 2))
] + [("zero_expert_mix", c) for c in MIX + (
    dict(y=0), dict(out=0), dict(out=A[2]), dict(out=A[3] + 2), dict(out=A[3], ld_out=65), dict(out=A[1]))
] + [("zero_expert_mix_backward", c) for c in MIX + (
    dict(dout=0), dict(y=0), dict(dweight=0), dict(dy=A[2]), dict(dy=A[3], ld_dy=65), dict(dweight=A[1]), dict(dweight=A[4]))
] + [("zero_log_probs", c) for c in ROWS + (
    dict(k=-1), dict(k=1025), dict(logp=0), dict(top_index=0), dict(top_logp=0), dict(logp=A[3]), dict(stats=A[0]),
    dict(entropy=A[3] + 1))
] + [("zero_log_probs_backward", c) for c in ROWS + (
    dict(grad_scale=NAN), dict(grad_scale=INF), dict(grad_scale=1e30, temperature=1e-20), dict(stats=0), dict(dlogp=0),
    dict(dlogits=0), dict(dlogits=A[0] + 4), dict(dlogits=A[0], ld_dlogits=1001), dict(dlogits=A[2]), dict(ld_dlogits=1))]


def call(zo, fn, **change):  # noqa: F811
    record, values = GOOD[fn]
    values = dict(values, **change)
    assert list(GOOD[fn][1]) == [n for _, n in fields(record)]
    return getattr(zo._lib, fn)(getattr(zo, RECORDS[record]).pack(*values.values()), None)


@pytest.mark.parametrize("fn,change", BAD, ids=lambda v: v if isinstance(v, str) else ",".join(v))
def test_wrong_arguments_are_refused(zo, fn, change):  # noqa: F811
    assert call(zo, fn, **change) == -1, change
    said = zo._lib.zero_last_error().decode()
    assert said.startswith((fn, "zero_expert_workspace")) and "GPU-accessible" not in said, said


@pytest.mark.parametrize("fn", sorted(GOOD))
def test_right_arguments_get_as_far_as_the_device(zo, fn):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("the addresses are not to reach a device")
    assert call(zo, fn) < 0
    assert "hip" in zo._lib.zero_last_error().decode()
    assert getattr(zo._lib, fn)(None, None) == -1


@pytest.mark.parametrize("fn,rows", (("zero_expert_product", "slots"), ("zero_expert_mix", "tokens"),
                                     ("zero_expert_mix_backward", "tokens"), ("zero_log_probs", "rows"),
                                     ("zero_log_probs_backward", "rows")))
def test_no_rows_need_no_device(zo, fn, rows):  # noqa: F811
    assert call(zo, fn, **{rows: 0}) == 0


def test_what_may_be_left_out_and_in_place(zo):  # noqa: F811
    if torch.cuda.is_available():
        pytest.skip("the addresses are not to reach a device")
    for fn, change in (("zero_expert_product", dict(x_slots=0, y_slots=0, order=0)),
                       ("zero_expert_product", dict(transposed=1, ld_weight=64)),
                       ("zero_expert_weight_backward", dict(x_slots=0, dy_slots=0, order=0)),
                       ("zero_expert_mix", dict(index=0, weight=0, base=0)), ("zero_expert_mix", dict(out=A[3])),
                       ("zero_expert_mix_backward", dict(index=0, weight=0, y=0, dweight=0)),
                       ("zero_expert_mix_backward", dict(dy=0)), ("zero_expert_mix_backward", dict(dy=A[3])),
                       ("zero_log_probs", dict(tokens=0, logp=0, entropy=0, stats=0)),
                       ("zero_log_probs", dict(k=0, top_index=0, top_logp=0)),
                       ("zero_log_probs_backward", dict(tokens=0, dlogp=0)),
                       ("zero_log_probs_backward", dict(dentropy=0, dlogits=A[0]))):
        assert call(zo, fn, **change) < 0
        assert "hip" in zo._lib.zero_last_error().decode(), (fn, change)


def test_workspace_sizes(zo):  # noqa: F811
    assert zo.zero_expert_workspace(0, 8, 64, 64) == 0
    for slots in (1, 1000, 10 ** 5, 2 ** 31 - 1):
        for experts, cin, cout in ((1, 1, 1), (8, 128, 256), (64, 4096, 1024), (1024, 1 << 20, 1 << 20)):
            assert 0 <= zo.zero_expert_workspace(slots, experts, cin, cout) <= 1 << 24
    for bad in ((-1, 8, 8, 8), (2 ** 31, 8, 8, 8), (8, 0, 8, 8), (8, 1025, 8, 8), (8, 8, 0, 8), (8, 8, 8, (1 << 20) + 1)):
        with pytest.raises(zo.ZeroError):
            zo.zero_expert_workspace(*bad)


def test_binding_refuses_host_tensors_and_wrong_types(zo):  # noqa: F811
    x, w, o = torch.zeros(4, 8), torch.zeros(2, 8, 8), torch.zeros(3, dtype=torch.int32)
    for call_ in (lambda: zo.zero_expert_product(x, w, o, x.clone()), lambda: zo.zero_expert_product(x.double(), w, o, x),
                  lambda: zo.zero_expert_weight_backward(x, x.clone(), o, w),
                  lambda: zo.zero_expert_mix(x, o, x.clone()), lambda: zo.zero_log_probs(x, None, None),
                  lambda: zo.zero_log_probs_backward(x, None, torch.zeros(4, 3), x.clone())):
        with pytest.raises((TypeError, ValueError)):
            call_()


# --- the checks themselves ---------------------------------------------------------

def test_plain_forms_agree_with_torch():
    z = C.normal(C.rng(3), 4, 30)
    tokens = torch.tensor([3, -1, 29, 30], dtype=torch.int32)
    got = L.log_probs(z, tokens, 5, 0.7)
    lp = torch.log_softmax(z / 0.7, 1)
    assert torch.allclose(got["logp"][0], torch.stack([lp[0, 3], lp[0, 0] * 0, lp[2, 29], lp[0, 0] * 0]), rtol=1e-12)
    assert torch.allclose(got["entropy"][0], torch.special.entr(lp.exp()).sum(1), rtol=1e-12)
    top = lp.topk(5, dim=1)
    assert torch.equal(got["top_index"], top.indices) and torch.allclose(got["top_logp"][0], top.values, rtol=1e-12)
    for name in ("logp", "entropy"):
        with pytest.raises(AssertionError):
            C.within(got[name][0] + 1e-3, *got[name], "planted")
    zv = z.clone().requires_grad_(True)
    a, b = torch.tensor([1.0, 2.0, -0.5, 3.0]), torch.tensor([0.3, -1.0, 2.0, 0.1])
    lv = torch.log_softmax(zv / 0.7, 1)
    loss = a[0] * lv[0, 3] + a[2] * lv[2, 29] + (b * torch.special.entr(lv.exp()).sum(1)).sum()
    want = torch.autograd.grad(loss * 8.0, zv)[0]
    g, bound = L.backward(z, tokens, a, b, 0.7, 8.0)
    assert torch.allclose(g, want, rtol=1e-9, atol=1e-12)
    C.within(g.float(), g, C.rounded(bound, g, torch.float32), "g")
    with pytest.raises(AssertionError):
        C.within(g * (1 + 1e-3), g, C.rounded(bound, g, torch.float32), "g")


def test_plain_experts_agree_with_torch_and_find_mistakes():
    index, offsets, placed = E.choice(20, 3, 4, 7, 0.2)
    g = C.rng(8)
    x, w = C.normal(g, 20, 6).requires_grad_(True), C.normal(g, 4, 6, 5).requires_grad_(True)
    flat = index.view(-1).long()
    y, bound, written = E.product(x.detach(), w.detach(), offsets, placed, 3, 1, False, 60)
    want = torch.einsum("sc,scn->sn", x[torch.arange(60) // 3], w[flat.clamp(min=0)]) * (flat >= 0)[:, None]
    assert torch.allclose(y, want.detach(), rtol=1e-12) and torch.equal(written, flat >= 0)
    dy = C.normal(g, 60, 5)
    gx, gw = torch.autograd.grad((want * dy).sum(), (x, w))
    dw, wb = E.weight_backward(x.detach(), dy, offsets, placed, 3, 1)
    assert torch.allclose(dw, gw, rtol=1e-12)
    dx, _, _ = E.product(dy, w.detach(), offsets, placed, 1, 1, True, 60)
    out, _ = E.mix(dx, index, None, None)
    assert torch.allclose(out, gx, rtol=1e-12)
    weight = torch.rand(20, 3, generator=g).requires_grad_(True)
    yv = y.clone().requires_grad_(True)
    mixed = (yv.view(20, 3, 5) * weight.double()[:, :, None] * (index >= 0)[:, :, None]).sum(1)
    assert torch.allclose(E.mix(y, index, weight.detach(), None)[0], mixed.detach(), rtol=1e-12)
    dout = C.normal(g, 20, 5)
    gy, gwt = torch.autograd.grad((mixed * dout).sum(), (yv, weight))
    dyy, dwt, _ = E.mix_backward(dout, y, index, weight.detach())
    assert torch.allclose(dyy, gy, rtol=1e-12) and torch.allclose(dwt.float(), gwt, rtol=1e-5)
    for wrong, right, b in ((y.roll(1, 0), y, bound), (dw * (1 + 1e-4), dw, wb)):
        with pytest.raises(AssertionError):
            C.within(wrong, right, b, "planted")
