"""The training operators' C ABI and binding without a GPU: what the header declares is exported, the records
are laid out alike in C and Python, wrong arguments are refused before any HIP call, and the checks that
the GPU tests use find a planted mistake."""
import math
import os
import re
import shutil
import subprocess
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_checks as C  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "zero_operators.h")
RECORDS = {"zero_rms_norm_args_t": "RMS_NORM_ARGS", "zero_rms_norm_backward_args_t": "RMS_NORM_BACKWARD_ARGS",
           "zero_route_args_t": "ROUTE_ARGS", "zero_route_order_args_t": "ROUTE_ORDER_ARGS",
           "zero_route_backward_args_t": "ROUTE_BACKWARD_ARGS", "zero_distill_args_t": "DISTILL_ARGS"}


@pytest.fixture(scope="module")
def zo():
    from paper_1910_02054_amd import build as b
    if b.is_stale():
        b.build()
    from paper_1910_02054_amd import operators
    return operators


def test_every_declared_call_is_exported(zo):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"^int (zero_\w+)\s*\(", text, flags=re.M))
    assert names == set(zo.EXPORTS)
    for n in names:
        assert hasattr(zo._lib, n)


def fields(record):
    """The members of a record in the header, in order: (C type, name)."""
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % record, text).group(1)
    out = []
    for line in body.split(";"):
        line = " ".join(line.split())
        if line:
            base, rest = re.match(r"((?:const )?\w+) ?(.*)", line).groups()
            out += [(base + ("*" if "*" in v else ""), v.strip("* ")) for v in rest.split(",")]
    return out


@pytest.mark.parametrize("record", sorted(RECORDS))
def test_records_have_the_headers_fields(zo, record):
    code = {"int32_t": "i", "int64_t": "q", "double": "d"}
    want = "".join("P" if t.endswith("*") else code[t] for t, _ in fields(record))
    assert getattr(zo, RECORDS[record]).format == "@" + want


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_records_have_the_compilers_sizes(zo, tmp_path):
    """Compiled as plain C99, which the header must be."""
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
    "zero_rms_norm": ("zero_rms_norm_args_t", dict(
        dtype=1, group=128, rows=4, cols=256, eps=1e-6, x=A[0], ld_x=256, residual=A[1], ld_residual=256, weight=A[2],
        h=A[3], ld_h=256, y=A[4], ld_y=256, q8=A[5], ld_q8=256, scale=A[6], rstd=A[7])),
    "zero_rms_norm_backward": ("zero_rms_norm_backward_args_t", dict(
        dtype=1, pad_=0, rows=4, cols=256, dy=A[0], ld_dy=256, h=A[1], ld_h=256, weight=A[2], rstd=A[3], dh=A[4],
        ld_dh=256, dx=A[5], ld_dx=256, dweight=A[6], workspace=A[7], workspace_floats=4096)),
    "zero_route": ("zero_route_args_t", dict(
        dtype=0, score=1, rows=4, experts=64, k=6, groups=8, top_groups=4, group_top=2, renormalise=1, scale=1.0,
        logits=A[0], ld_logits=64, bias=A[1], index=A[2], weight=A[3])),
    "zero_route_order": ("zero_route_order_args_t", dict(
        index=A[0], slots=10000, experts=64, pad_=0, offsets=A[1], order=A[2], workspace=A[3], workspace_ints=1 << 20)),
    "zero_route_backward": ("zero_route_backward_args_t", dict(
        dtype=0, score=0, rows=4, experts=64, k=6, renormalise=1, pad_=0, scale=1.0, logits=A[0], ld_logits=64,
        bias=A[1], index=A[2], dweight=A[3], dlogits=A[4], ld_dlogits=64)),
    "zero_distill_step": ("zero_distill_args_t", dict(
        dtype=2, teacher_dtype=1, rows=4, vocab=1000, k=8, pad_=0, temperature=2.0, soft=1.0, hard=0.5, grad_scale=64.0,
        logits=A[0], ld_logits=1000, teacher_index=A[1], teacher_logits=A[2], labels=A[3], row_weight=A[4], loss=A[5],
        stats=0, dloss=0, dlogits=A[6], ld_dlogits=1000)),
    "zero_distill_loss": ("zero_distill_args_t", dict(
        dtype=2, teacher_dtype=1, rows=4, vocab=1000, k=8, pad_=0, temperature=2.0, soft=1.0, hard=0.5, grad_scale=64.0,
        logits=A[0], ld_logits=1000, teacher_index=A[1], teacher_logits=A[2], labels=A[3], row_weight=A[4], loss=A[5],
        stats=A[7], dloss=0, dlogits=0, ld_dlogits=0)),
    "zero_distill_backward": ("zero_distill_args_t", dict(
        dtype=2, teacher_dtype=1, rows=4, vocab=1000, k=8, pad_=0, temperature=2.0, soft=1.0, hard=0.5, grad_scale=64.0,
        logits=A[0], ld_logits=1000, teacher_index=A[1], teacher_logits=A[2], labels=A[3], row_weight=A[4], loss=0,
        stats=A[7], dloss=A[8], dlogits=A[6], ld_dlogits=1000)),
}
NAN, INF = math.nan, math.inf
BAD = [
    ("zero_rms_norm", c) for c in (
        dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=(1 << 40) + 1), dict(cols=0), dict(cols=32769),
        dict(eps=-1e-6), dict(eps=NAN), dict(eps=INF), dict(group=16), dict(group=-1), dict(group=512), dict(q8=0),
        dict(scale=0), dict(residual=0), dict(x=0), dict(weight=0), dict(x=A[0] + 1), dict(scale=A[6] + 2),
        dict(rstd=A[7] + 1), dict(ld_x=255), dict(ld_y=100), dict(ld_q8=-1), dict(y=A[0] + 2), dict(y=A[0], ld_y=300),
        dict(h=A[4]), dict(q8=A[0]), dict(rstd=A[2]), dict(y=A[1] + 2 * 300), dict(ld_x=1 << 41),
        dict(y=A[0] + 256, ld_y=300, ld_x=300))
] + [
    ("zero_rms_norm_backward", c) for c in (
        dict(dtype=7), dict(rows=-5), dict(cols=0), dict(cols=40000), dict(dy=0), dict(h=0), dict(weight=0), dict(rstd=0),
        dict(dx=0), dict(dweight=0), dict(workspace=0), dict(workspace_floats=1023), dict(workspace_floats=-1),
        dict(dx=A[0] + 2), dict(dx=A[2]), dict(dweight=A[2]), dict(workspace=A[5]), dict(ld_dh=3), dict(rstd=A[3] + 2))
] + [
    ("zero_route", c) for c in (
        dict(dtype=9), dict(score=2), dict(score=-1), dict(rows=-1), dict(experts=0), dict(experts=1025), dict(k=0),
        dict(k=65), dict(k=7, experts=6, groups=1, top_groups=1), dict(groups=0), dict(groups=7), dict(groups=65),
        dict(top_groups=0), dict(top_groups=9), dict(group_top=0), dict(group_top=3),
        dict(groups=64, top_groups=4), dict(scale=NAN), dict(scale=INF), dict(rows=1 << 30), dict(logits=0), dict(index=0),
        dict(weight=0), dict(ld_logits=63), dict(index=A[0]), dict(weight=A[2]), dict(bias=A[1] + 2))
] + [
    ("zero_route_order", c) for c in (
        dict(slots=-1), dict(slots=1 << 31), dict(experts=0), dict(experts=1025), dict(index=0), dict(offsets=0),
        dict(order=0), dict(workspace=0), dict(workspace_ints=10), dict(order=A[0]), dict(order=A[0] + 4),
        dict(offsets=A[3]), dict(index=A[0] + 1))
] + [
    ("zero_route_backward", c) for c in (
        dict(dtype=5), dict(score=3), dict(rows=-1), dict(experts=0), dict(k=0), dict(k=65), dict(scale=NAN), dict(logits=0),
        dict(index=0), dict(dweight=0), dict(dlogits=0), dict(ld_dlogits=10), dict(dlogits=A[0] + 4), dict(dlogits=A[3]),
        dict(dlogits=A[0], ld_dlogits=65))
] + [
    (f, c) for f in ("zero_distill_step", "zero_distill_loss", "zero_distill_backward") for c in (
        dict(dtype=3), dict(teacher_dtype=4), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(k=-1),
        dict(k=1025), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-31),
        dict(temperature=1e31),
        dict(soft=NAN), dict(hard=INF), dict(grad_scale=NAN), dict(logits=0), dict(teacher_index=0),
        dict(teacher_logits=0), dict(ld_logits=999), dict(logits=A[0] + 1), dict(labels=A[3] + 2))
] + [
    ("zero_distill_step", c) for c in (dict(loss=0), dict(dlogits=0), dict(stats=A[7]), dict(dloss=A[8]),
                                       dict(dlogits=A[0] + 2), dict(dlogits=A[0], ld_dlogits=1008), dict(dlogits=A[1]),
                                       dict(loss=A[4]))
] + [
    ("zero_distill_loss", c) for c in (dict(loss=0), dict(dlogits=A[6], ld_dlogits=1000), dict(dloss=A[8]),
                                       dict(stats=A[5]))
] + [("zero_distill_backward", c) for c in (dict(loss=A[5]), dict(dlogits=0), dict(stats=0), dict(dlogits=A[7]))]


def call(zo, fn, **change):
    record, values = GOOD[fn]
    values = dict(values, **change)
    assert list(GOOD[fn][1]) == [n for _, n in fields(record)]
    return getattr(zo._lib, fn)(getattr(zo, RECORDS[record]).pack(*values.values()), None)


@pytest.mark.parametrize("fn,change", BAD, ids=lambda v: v if isinstance(v, str) else ",".join(v))
def test_wrong_arguments_are_refused(zo, fn, change):
    assert call(zo, fn, **change) == -1, change
    said = zo._lib.zero_last_error().decode()
    assert said.startswith((fn, "zero_rms_norm_workspace", "zero_route_workspace")) and "GPU-accessible" not in said, said


@pytest.mark.parametrize("fn", sorted(GOOD))
def test_right_arguments_get_as_far_as_the_device(zo, fn):
    """Without a GPU the good record fails too, but only once its arguments have been taken."""
    if torch.cuda.is_available():
        pytest.skip("the addresses are not to reach a device")
    assert call(zo, fn) < 0
    assert "hip" in zo._lib.zero_last_error().decode()


@pytest.mark.parametrize("fn", sorted(GOOD))
def test_null_record_is_refused(zo, fn):
    assert getattr(zo._lib, fn)(None, None) == -1


@pytest.mark.parametrize("fn", ("zero_rms_norm", "zero_route", "zero_route_backward", "zero_distill_step",
                                "zero_distill_loss", "zero_distill_backward"))
def test_no_rows_need_no_device(zo, fn):
    assert call(zo, fn, rows=0) == 0


def test_in_place_and_columns_of_one_buffer_are_taken(zo):
    if torch.cuda.is_available():
        pytest.skip("the addresses are not to reach a device")
    for fn, change in (("zero_rms_norm", dict(h=A[1])), ("zero_rms_norm", dict(h=A[0])), ("zero_rms_norm", dict(y=A[0])),
                       ("zero_rms_norm", dict(y=A[0] + 512, ld_y=512, ld_x=512)),
                       ("zero_rms_norm_backward", dict(dx=A[0])), ("zero_rms_norm_backward", dict(dx=A[1])),
                       ("zero_rms_norm_backward", dict(dx=A[4])), ("zero_route_backward", dict(dlogits=A[0])),
                       ("zero_distill_step", dict(dlogits=A[0])), ("zero_distill_backward", dict(dlogits=A[0]))):
        call(zo, fn, **change)
        assert "overlap" not in zo._lib.zero_last_error().decode(), (fn, change)


def test_workspace_sizes(zo):
    assert zo.zero_rms_norm_workspace(0, 100) == zo.zero_rms_norm_workspace(1, 100) == 0
    for rows in (2, 255, 256, 10 ** 6):
        assert 0 < zo.zero_rms_norm_workspace(rows, 100) <= 1024 * 100
    for rows, cols in ((-1, 10), (10, 0), (10, 32769)):
        with pytest.raises(zo.ZeroError):
            zo.zero_rms_norm_workspace(rows, cols)
    assert zo.zero_route_workspace(0, 8) == zo.zero_route_workspace(2048, 8) == 0
    for slots in (2049, 65535, 65536, 2 ** 31 - 1):
        assert 0 < zo.zero_route_workspace(slots, 8) <= 1024 * 9
    for slots, experts in ((-1, 8), (2 ** 31, 8), (10, 0), (10, 1025)):
        with pytest.raises(zo.ZeroError):
            zo.zero_route_workspace(slots, experts)


def test_binding_refuses_host_tensors_and_wrong_types(zo):
    x, w = torch.zeros(2, 8), torch.zeros(8)
    with pytest.raises(TypeError):
        zo.zero_rms_norm(x, w, 1e-6, y=x.clone())
    with pytest.raises(TypeError):
        zo.zero_rms_norm(x.double(), w, 1e-6)
    with pytest.raises(TypeError):
        zo.zero_distill_step(x, None, None, torch.zeros(2), x.clone())
    with pytest.raises(TypeError):
        zo.zero_route_order(torch.zeros(4), 3, torch.zeros(4), torch.zeros(4))
    with pytest.raises(ValueError):
        zo._score("relu")


# --- the checks themselves: a mistake planted in the plain implementation's result is found -------------

def test_checks_find_planted_mistakes():
    g = C.rng(1)
    h, w = C.normal(g, 4, 300), C.normal(g, 300)
    rstd, y = C.rms_norm(h, w, 1e-6)
    bound = C.rounded((C.ROOT + 8 * C.U) * y.abs(), y, torch.float16)
    C.within(y.half(), y, bound, "y")
    off = y.clone()
    off[2, 7] *= 1 + 2.0 ** -9                 # two units of fp16
    with pytest.raises(AssertionError):
        C.within(off.half(), y, bound, "y")
    off = y.clone()
    off[1, 1] = math.nan
    with pytest.raises(AssertionError):
        C.within(off, y, bound, "y")
    q = (y / C.spread(C.scales(y, 64), 300, 64)).float().to(torch.float8_e4m3fn).view(torch.uint8)
    C.check_e4m3(q, y, 64, "q8")
    q[0, 5] ^= 1
    with pytest.raises(AssertionError):
        C.check_e4m3(q, y, 64, "q8")
    z = C.normal(g, 3, 50)
    index = torch.tensor([[1, 4], [2, -1], [7, 7]], dtype=torch.int32)
    t = C.normal(g, 3, 2)
    loss, lb, d, db = C.distill(z, index, t, None, 1.0, 0.0, 2.0, None, 1.0)
    C.within(d.float(), d, C.rounded(db, d, torch.float32), "d")
    for wrong in (d * (1 + 1e-4), d.roll(1, 1)):
        with pytest.raises(AssertionError):
            C.within(wrong, d, C.rounded(db, d, torch.float32), "d")
    with pytest.raises(AssertionError):
        C.within(loss * (1 + 1e-3), loss, lb, "loss")


def test_plain_gradients_agree_with_autograd():
    """The written-out derivatives of operator_checks against automatic differentiation of the forwards."""
    g = C.rng(2)
    h, w, dy = C.normal(g, 3, 20), C.normal(g, 20), C.normal(g, 3, 20)
    hv, wv = h.clone().requires_grad_(True), w.clone().requires_grad_(True)
    rstd = (hv.square().mean(1) + 1e-6).rsqrt()
    gh, gw = torch.autograd.grad((hv * rstd[:, None] * wv * dy).sum(), (hv, wv))
    dx, dw, _, _ = C.rms_norm_backward(dy, h, w, rstd.detach(), None)
    assert torch.allclose(dx, gh, rtol=1e-10, atol=1e-12) and torch.allclose(dw, gw, rtol=1e-10, atol=1e-12)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            z, d = C.normal(g, 4, 9), C.normal(g, 4, 3)
            index, _, _ = C.route(z, None, score, 1, 1, 1, 3, renorm, 1.5)
            zv = z.clone().requires_grad_(True)
            wt = C.weights(zv, torch.zeros_like(z, dtype=torch.bool), index, score, renorm, 1.5)
            want = torch.autograd.grad((wt * d).sum(), zv)[0]
            got, _ = C.route_backward(z, None, index, d, score, renorm, 1.5)
            assert torch.allclose(got, want, rtol=1e-9, atol=1e-12)
    z = C.normal(g, 3, 30)
    index = torch.tensor([[1, 4, 9], [2, -1, 5], [7, 8, 7]], dtype=torch.int32)
    t, labels = C.normal(g, 3, 3), torch.tensor([4, -1, 0], dtype=torch.int32)
    weight, up = torch.rand(3, generator=g), torch.rand(3, generator=g)
    zv = z.clone().requires_grad_(True)
    absent = index < 0
    p = torch.softmax((t / 1.5).masked_fill(absent, -math.inf), 1)
    lq, l1 = torch.log_softmax(zv / 1.5, 1), torch.log_softmax(zv, 1)
    at = index.long().clamp(min=0)
    each = torch.where(absent, 0.0, p * (torch.log(p.clamp(min=1e-300)) - lq.gather(1, at)))
    hard = torch.where(labels >= 0, -l1.gather(1, labels.long().clamp(min=0)[:, None])[:, 0], 0.0)
    loss = weight.double() * (0.7 * 1.5 ** 2 * each.sum(1) + 0.3 * hard)
    want = torch.autograd.grad((loss * up.double()).sum() * 8.0, zv)[0]
    got_loss, _, got, _ = C.distill(z, index, t, labels, 0.7, 0.3, 1.5, weight, 8.0, up)
    assert torch.allclose(got_loss, loss.detach(), rtol=1e-10) and torch.allclose(got, want, rtol=1e-9, atol=1e-12)
