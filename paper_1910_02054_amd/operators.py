"""Thin ctypes binding of the training operators of ``libzeroshard.so`` (C ABI in
``include/zero_operators.h``).

As in ``binding``: argument marshalling only, every operator runs in the library's HIP
kernels, outputs are tensors of the caller's, calls only enqueue work on torch's current
stream (or `stream`) and can be captured into a graph, and ZeroError carries the library's
message.  Matrices are torch tensors on the current device whose last dimension is contiguous; leading
dimensions are taken as one where their strides allow it, else the rows may be any stride
apart.
"""
import ctypes
import struct

import torch

from .binding import ZeroError, _check, _lib, _stream  # noqa: F401

ZERO_F32, ZERO_F16, ZERO_BF16 = 0, 1, 2
ZERO_SCORE_SOFTMAX, ZERO_SCORE_SIGMOID = 0, 1
_TYPE = {torch.float32: ZERO_F32, torch.float16: ZERO_F16, torch.bfloat16: ZERO_BF16}
_SCORE = {"softmax": ZERO_SCORE_SOFTMAX, "sigmoid": ZERO_SCORE_SIGMOID}

_P, _i64, _i32, _dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double


# The argument records of the C ABI (zero_rms_norm_args_t and so on), their fields in order: packed
# into bytes for the call, which takes half the time of filling a ctypes.Structure of that many fields.
RMS_NORM_ARGS = struct.Struct("@iiqqdPqPqPPqPqPqPP")
RMS_NORM_BACKWARD_ARGS = struct.Struct("@iiqqPqPqPPPqPqPPq")
ROUTE_ARGS = struct.Struct("@iiqiiiiiidPqPPP")
ROUTE_ORDER_ARGS = struct.Struct("@PqiiPPPq")
ROUTE_BACKWARD_ARGS = struct.Struct("@iiqiiiidPqPPPPq")
DISTILL_ARGS = struct.Struct("@iiqqiiddddPqPPPPPPPPq")

EXPORTS = ("zero_rms_norm", "zero_rms_norm_backward", "zero_rms_norm_workspace", "zero_route", "zero_route_order",
           "zero_route_workspace", "zero_route_backward", "zero_distill_step", "zero_distill_loss",
           "zero_distill_backward")
for _f in EXPORTS:
    getattr(_lib, _f).restype = ctypes.c_int
    getattr(_lib, _f).argtypes = [_P, _P]
_lib.zero_rms_norm_workspace.argtypes = [_i64, _i64, ctypes.POINTER(_i64)]
_lib.zero_route_workspace.argtypes = [_i64, _i32, ctypes.POINTER(_i64)]


_raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _on(stream, dev=None):
    """The hipStream_t of `stream`, or of torch's current stream on the current device, which must be `dev`, the
    device of a call's tensors."""
    if dev is not None:
        if dev < 0:
            raise TypeError("a call's arrays must be device tensors")
        here = _device()
        if dev != here:
            raise ValueError("the tensors are on device %d, the current device is %d" % (dev, here))
        if stream is None:
            return _raw_stream(here)
    return _raw_stream(_device()) if stream is None else _stream(stream)


def _elsewhere(t, what, dev):
    """The error of a tensor that is not on `dev`, where the call's first one is (-1: the host)."""
    at = t.get_device()
    if at < 0 or dev < 0:
        return TypeError("%s: a call's arrays must be device tensors" % what)
    return ValueError("%s is on device %d, other tensors of the call on device %d" % (what, at, dev))


def _type(t, what):
    code = _TYPE.get(getattr(t, "dtype", None))
    if code is None:
        raise TypeError("%s must be a tensor of one of %s" % (what, tuple(_TYPE)))
    return code


def _sizes(t, what):
    """(rows, columns) of a matrix whose leading dimensions count as one."""
    shape = t.shape
    if len(shape) == 2:
        return shape
    if not shape:
        raise ValueError("%s must have a dimension" % what)
    n = shape[-1]
    return torch.Size((t.numel() // n if n else 0, n))


def _matrix(t, dtype, what, size, dev):
    """(address, elements from row to row) of a matrix of the given type and size on device `dev`; (0, cols) for
    None."""
    if t is None:
        return 0, size[1]
    if t.dtype is not dtype:
        raise TypeError("%s: dtype %s, not %s" % (what, t.dtype, dtype))
    if t.get_device() != dev:
        raise _elsewhere(t, what, dev)
    if t.shape != size:
        if _sizes(t, what) != size:
            raise ValueError("%s has shape %s, not %s" % (what, list(t.shape), list(size)))
        t = t.view(size) if t.numel() else t.reshape(size)
    step, one = t.stride()
    rows, cols = size
    if one != 1 and cols > 1 and rows > 0:
        raise ValueError("%s: the last dimension must be contiguous" % what)
    return t.data_ptr(), step if rows > 1 else cols


def _vector(t, dtype, what, numel, dev):
    """The address of a contiguous array of `numel` elements on device `dev` (0 for None)."""
    if t is None:
        return 0
    if t.dtype is not dtype:
        raise TypeError("%s: dtype %s, not %s" % (what, t.dtype, dtype))
    if t.get_device() != dev:
        raise _elsewhere(t, what, dev)
    if not t.is_contiguous():
        raise TypeError("%s must be contiguous" % what)
    if t.numel() != numel:
        raise ValueError("%s has %d elements, not %d" % (what, t.numel(), numel))
    return t.data_ptr()


def _room(t, dtype, what, dev):
    """(address, elements) of a workspace, which may be None."""
    return (0, 0) if t is None else (_vector(t, dtype, what, t.numel(), dev), t.numel())


_F32, _I32 = torch.float32, torch.int32


def zero_rms_norm(x, weight, eps, residual=None, h=None, y=None, q8=None, scale=None, group=0, rstd=None,
                  stream=None):
    """h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h * rstd * weight, and with q8 and scale the
    rows y in e4m3 (torch.float8_e4m3fn or uint8 codes) with one fp32 scale for each `group` columns (0: a row).
    Each output is written where a tensor is given; y, q8 * scale and h are [rows, cols], rstd [rows],
    scale [rows, ceil(cols / group)].  h may be residual or x in place, and so may y."""
    code, dt = _type(x, "x"), x.dtype
    dev = x.get_device()
    size = rows, cols = _sizes(x, "x")
    px, ld_x = _matrix(x, dt, "x", size, dev)
    pr, ld_r = _matrix(residual, dt, "residual", size, dev)
    ph, ld_h = _matrix(h, dt, "h", size, dev)
    py, ld_y = _matrix(y, dt, "y", size, dev)
    pq, ld_q, ps = 0, cols, 0
    if q8 is not None:
        pq, ld_q = _matrix(q8, torch.uint8 if q8.dtype is torch.uint8 else torch.float8_e4m3fn, "q8", size, dev)
    if scale is not None:
        ps = _vector(scale, _F32, "scale", rows * (-(-cols // group) if group > 0 else 1), dev)
    pw, prs = _vector(weight, dt, "weight", cols, dev), _vector(rstd, _F32, "rstd", rows, dev)
    args = RMS_NORM_ARGS.pack(code, group, rows, cols, eps, px, ld_x, pr, ld_r, pw, ph, ld_h, py, ld_y, pq, ld_q, ps,
                              prs)
    rc = _lib.zero_rms_norm(args, _on(stream, dev))
    if rc < 0:
        _check(rc)


def zero_rms_norm_workspace(rows, cols):
    """Floats of workspace that zero_rms_norm_backward needs for these sizes (at most 1024 * cols)."""
    out = _i64()
    _check(_lib.zero_rms_norm_workspace(int(rows), int(cols), ctypes.byref(out)))
    return out.value


def zero_rms_norm_backward(dy, h, weight, rstd, dx, dweight, workspace=None, dh=None, stream=None):
    """The gradients of zero_rms_norm into dx [rows, cols] (of x and of the residual alike; may be dy, h or dh in
    place) and dweight [cols], from dy, the h and rstd of the forward (h is x where it had no residual) and the
    gradient dh that reaches h from elsewhere.  workspace: a float32 tensor of at least
    zero_rms_norm_workspace(rows, cols) elements."""
    code, dt = _type(h, "h"), h.dtype
    dev = h.get_device()
    size = rows, cols = _sizes(h, "h")
    ph, ld_h = _matrix(h, dt, "h", size, dev)
    pdy, ld_dy = _matrix(dy, dt, "dy", size, dev)
    pdh, ld_dh = _matrix(dh, dt, "dh", size, dev)
    pdx, ld_dx = _matrix(dx, dt, "dx", size, dev)
    pw, n = _room(workspace, _F32, "workspace", dev)
    args = RMS_NORM_BACKWARD_ARGS.pack(code, 0, rows, cols, pdy, ld_dy, ph, ld_h,
                                       _vector(weight, dt, "weight", cols, dev), _vector(rstd, _F32, "rstd", rows, dev),
                                       pdh, ld_dh, pdx, ld_dx, _vector(dweight, dt, "dweight", cols, dev), pw, n)
    rc = _lib.zero_rms_norm_backward(args, _on(stream, dev))
    if rc < 0:
        _check(rc)


def _score(score):
    code = _SCORE.get(score)
    if code is None:
        raise ValueError("score must be one of %s" % (tuple(_SCORE),))
    return code


def zero_route(logits, index, weight, score="softmax", bias=None, groups=1, top_groups=1, group_top=1,
               renormalise=True, scale=1.0, stream=None):
    """The choice of k experts for each row of logits [tokens, experts]: index (int32) and weight (float32), both
    [tokens, k], in falling order of the keys.  score: "softmax" or "sigmoid"; bias [experts] float32 acts on the
    choice alone; groups > 1 keeps the top_groups groups of the largest sums of their group_top largest keys."""
    code = _type(logits, "logits")
    dev = logits.get_device()
    size = rows, experts = _sizes(logits, "logits")
    pl, ld = _matrix(logits, logits.dtype, "logits", size, dev)
    k = index.shape[-1]
    args = ROUTE_ARGS.pack(code, _score(score), rows, experts, k, groups, top_groups, group_top, bool(renormalise),
                           scale, pl, ld, _vector(bias, _F32, "bias", experts, dev),
                           _vector(index, _I32, "index", rows * k, dev), _vector(weight, _F32, "weight", rows * k, dev))
    rc = _lib.zero_route(args, _on(stream, dev))
    if rc < 0:
        _check(rc)


def zero_route_workspace(slots, experts):
    """Ints of workspace that zero_route_order needs for these sizes (at most 1024 * (experts + 1))."""
    out = _i64()
    _check(_lib.zero_route_workspace(int(slots), int(experts), ctypes.byref(out)))
    return out.value


def zero_route_order(index, experts, offsets, order, workspace=None, stream=None):
    """The slots (flat positions in index, int32) by expert, then by slot: order[offsets[e]:offsets[e + 1]] are
    expert e's; slots without an expert are left out and order ends in as many -1.  offsets [experts + 1] and order
    [slots] are int32; workspace: int32, at least zero_route_workspace(slots, experts) elements."""
    n, dev = index.numel(), index.get_device()
    pw, room = _room(workspace, _I32, "workspace", dev)
    args = ROUTE_ORDER_ARGS.pack(_vector(index, _I32, "index", n, dev), n, experts, 0,
                                 _vector(offsets, _I32, "offsets", experts + 1, dev),
                                 _vector(order, _I32, "order", n, dev), pw, room)
    rc = _lib.zero_route_order(args, _on(stream, dev))
    if rc < 0:
        _check(rc)


def zero_route_backward(logits, index, dweight, dlogits, score="softmax", bias=None, renormalise=True, scale=1.0,
                        stream=None):
    """The gradient of zero_route's logits into dlogits [tokens, experts] (may be logits in place) from that of its
    weights, dweight [tokens, k] float32, and its index."""
    code, dt = _type(logits, "logits"), logits.dtype
    dev = logits.get_device()
    size = rows, experts = _sizes(logits, "logits")
    pl, ld = _matrix(logits, dt, "logits", size, dev)
    pd, ld_d = _matrix(dlogits, dt, "dlogits", size, dev)
    k = index.shape[-1]
    args = ROUTE_BACKWARD_ARGS.pack(code, _score(score), rows, experts, k, bool(renormalise), 0, scale, pl, ld,
                                    _vector(bias, _F32, "bias", experts, dev),
                                    _vector(index, _I32, "index", rows * k, dev),
                                    _vector(dweight, _F32, "dweight", rows * k, dev), pd, ld_d)
    rc = _lib.zero_route_backward(args, _on(stream, dev))
    if rc < 0:
        _check(rc)


def _distill(fn, logits, teacher_index, teacher_logits, loss, stats, dlogits, dloss, labels, soft, hard, temperature,
             row_weight, grad_scale, stream):
    code, dt = _type(logits, "logits"), logits.dtype
    dev = logits.get_device()
    size = rows, vocab = _sizes(logits, "logits")
    pl, ld = _matrix(logits, dt, "logits", size, dev)
    pd, ld_d = _matrix(dlogits, dt, "dlogits", size, dev)
    k, teacher, pi, pt = 0, ZERO_F32, 0, 0
    if teacher_index is not None:
        k = teacher_index.shape[-1]
        teacher = _type(teacher_logits, "teacher_logits")
        pi = _vector(teacher_index, _I32, "teacher_index", rows * k, dev)
        pt = _vector(teacher_logits, teacher_logits.dtype, "teacher_logits", rows * k, dev)
    args = DISTILL_ARGS.pack(code, teacher, rows, vocab, k, 0, temperature, soft, hard, grad_scale, pl, ld, pi, pt,
                             _vector(labels, _I32, "labels", rows, dev),
                             _vector(row_weight, _F32, "row_weight", rows, dev), _vector(loss, _F32, "loss", rows, dev),
                             _vector(stats, _F32, "stats", 3 * rows, dev), _vector(dloss, _F32, "dloss", rows, dev),
                             pd, ld_d)
    rc = fn(args, _on(stream, dev))
    if rc < 0:
        _check(rc)


def zero_distill_step(logits, teacher_index, teacher_logits, loss, dlogits, labels=None, soft=1.0, hard=0.0,
                      temperature=1.0, row_weight=None, grad_scale=1.0, stream=None):
    """Loss (float32, [rows]) and gradient (dlogits, like logits; may be logits in place) of student logits
    [rows, vocab] against a teacher's top logits: teacher_index (int32) and teacher_logits, both [rows, k], entries
    outside the vocabulary or of logit -inf absent.  hard weighs the cross entropy with `labels` (int32, outside the
    vocabulary: none).  grad_scale is the loss scale; row_weight [rows] float32 (0: the row is not looked at)."""
    _distill(_lib.zero_distill_step, logits, teacher_index, teacher_logits, loss, None, dlogits, None, labels, soft,
             hard, temperature, row_weight, grad_scale, stream)


def zero_distill_loss(logits, teacher_index, teacher_logits, loss, labels=None, soft=1.0, hard=0.0, temperature=1.0,
                      row_weight=None, stats=None, stream=None):
    """The loss alone, as zero_distill_step's; stats (float32, [rows, 3]) is what zero_distill_backward needs of it."""
    _distill(_lib.zero_distill_loss, logits, teacher_index, teacher_logits, loss, stats, None, None, labels, soft,
             hard, temperature, row_weight, 1.0, stream)


def zero_distill_backward(logits, teacher_index, teacher_logits, stats, dlogits, dloss=None, labels=None, soft=1.0,
                          hard=0.0, temperature=1.0, row_weight=None, grad_scale=1.0, stream=None):
    """The gradient of the logits from zero_distill_loss's stats (same other arguments) and the losses' gradient
    dloss (float32, [rows]; None: 1)."""
    _distill(_lib.zero_distill_backward, logits, teacher_index, teacher_logits, None, stats, dlogits, dloss, labels,
             soft, hard, temperature, row_weight, grad_scale, stream)
