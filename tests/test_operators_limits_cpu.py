"""What the training operators' calls refuse beside test_operators_cpu.py, without a GPU."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_operators_cpu as T  # noqa: E402


@pytest.fixture(scope="module")
def zo():
    from paper_1910_02054_amd import build as b
    if b.is_stale():
        b.build()
    from paper_1910_02054_amd import operators
    return operators


# --- scalars that fp32, in which the kernels have them, cannot hold ------------------------

TOO_LARGE = [("zero_route", dict(scale=4e38)), ("zero_route", dict(scale=-1e300)), ("zero_route_backward", dict(scale=4e38))] + [
    (f, c) for f in ("zero_distill_step", "zero_distill_loss", "zero_distill_backward") for c in (
        dict(soft=4e38, temperature=1.0), dict(soft=1e9, temperature=1e30), dict(soft=-1e300), dict(hard=4e38),
        dict(hard=-math.inf), dict(grad_scale=1e39))]


@pytest.mark.parametrize("fn,change", TOO_LARGE, ids=lambda v: v if isinstance(v, str) else ",".join(v))
def test_scalars_past_fp32_are_refused(zo, fn, change):
    assert T.call(zo, fn, **change) == -1
    said = zo._lib.zero_last_error().decode()
    assert said.startswith(fn) and "finite in fp32" in said


def test_scalars_at_fp32s_largest_are_taken(zo):
    for fn, change in (("zero_route", dict(scale=3.4e38)), ("zero_distill_step", dict(soft=1e8, temperature=1e30)),
                       ("zero_distill_step", dict(hard=-3.4e38, grad_scale=3.4e38))):
        assert T.call(zo, fn, rows=0, **change) == 0


# --- tensors of another device --------------------------------------------------------------

class At:
    """A host tensor that says it is on a device (the calls below are refused before they reach the library)."""

    def __init__(self, t, device=0):
        self.t, self.device_index, self.is_cuda = t, device, device >= 0

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.device_index


def all_calls(zo):
    """For each call of the binding, the function and its tensors by name."""
    f16, f32, i32 = torch.float16, torch.float32, torch.int32

    def e(dtype, *shape):
        return torch.empty(*shape, dtype=dtype)

    x = {n: e(f16, 4, 64) for n in ("x", "residual", "h", "y", "dy", "dh", "dx", "logits", "dlogits")}
    distill = dict(logits=x["logits"], teacher_index=e(i32, 4, 3), teacher_logits=e(f32, 4, 3), labels=e(i32, 4),
                   row_weight=e(f32, 4))
    return [
        (zo.zero_rms_norm, dict({n: x[n] for n in ("x", "residual", "h", "y")}, weight=e(f16, 64), rstd=e(f32, 4),
                                q8=e(torch.uint8, 4, 64), scale=e(f32, 4)), dict(eps=1e-6)),
        (zo.zero_rms_norm_backward, dict({n: x[n] for n in ("dy", "h", "dh", "dx")}, weight=e(f16, 64), rstd=e(f32, 4),
                                         dweight=e(f16, 64), workspace=e(f32, 256)), {}),
        (zo.zero_route, dict(logits=x["logits"], index=e(i32, 4, 2), weight=e(f32, 4, 2), bias=e(f32, 64)), {}),
        (zo.zero_route_order, dict(index=e(i32, 8), offsets=e(i32, 65), order=e(i32, 8), workspace=e(i32, 65)),
         dict(experts=64)),
        (zo.zero_route_backward, dict(logits=x["logits"], index=e(i32, 4, 2), dweight=e(f32, 4, 2),
                                      dlogits=x["dlogits"], bias=e(f32, 64)), {}),
        (zo.zero_distill_step, dict(distill, loss=e(f32, 4), dlogits=x["dlogits"]), {}),
        (zo.zero_distill_loss, dict(distill, loss=e(f32, 4), stats=e(f32, 4, 3)), {}),
        (zo.zero_distill_backward, dict(distill, stats=e(f32, 4, 3), dlogits=x["dlogits"], dloss=e(f32, 4)), {}),
    ]


def test_tensors_of_another_device_are_refused(zo, monkeypatch):
    monkeypatch.setattr(zo, "_device", lambda: 0)
    monkeypatch.setattr(zo, "_raw_stream", lambda d: 0)

    class Reached(Exception):
        pass

    def reached(*_):
        raise Reached

    monkeypatch.setattr(zo, "_lib", type("Lib", (), {f: staticmethod(reached) for f in zo.EXPORTS}))
    for fn, tensors, rest in all_calls(zo):
        with pytest.raises(Reached):
            fn(**{n: At(t) for n, t in tensors.items()}, **rest)
        for other in tensors:
            with pytest.raises(ValueError, match="device 1"):
                fn(**{n: At(t, int(n == other)) for n, t in tensors.items()}, **rest)
            with pytest.raises(TypeError, match="device tensor"):
                fn(**{n: At(t, -1 if n == other else 0) for n, t in tensors.items()}, **rest)
        with pytest.raises(ValueError, match="current device is 0"):
            fn(**{n: At(t, 1) for n, t in tensors.items()}, **rest)
