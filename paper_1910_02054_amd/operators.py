"""Thin ctypes binding of the training operators of ``libzeroshard.so`` (C ABI in
``include/zero_operators.h``).

As in ``binding``: argument marshalling only, every operator runs in the library's HIP
kernels, outputs are tensors of the caller's, calls only enqueue work on torch's current
stream (or `stream`) and can be captured into a graph, and ZeroError carries the library's
message.  Matrices are torch device tensors whose last dimension is contiguous; leading
dimensions are taken as one where their strides allow it, else the rows may be any stride
apart.
"""
import ctypes

import torch

from .binding import ZeroError, _addr, _check, _lib, _stream  # noqa: F401

ZERO_F32, ZERO_F16, ZERO_BF16 = 0, 1, 2
ZERO_SCORE_SOFTMAX, ZERO_SCORE_SIGMOID = 0, 1
_TYPE = {torch.float32: ZERO_F32, torch.float16: ZERO_F16, torch.bfloat16: ZERO_BF16}
_SCORE = {"softmax": ZERO_SCORE_SOFTMAX, "sigmoid": ZERO_SCORE_SIGMOID}
_Q8 = (torch.float8_e4m3fn, torch.uint8)

_P, _i64, _i32, _dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double


class RmsNormArgs(ctypes.Structure):
    """Mirror of zero_rms_norm_args_t."""
    _fields_ = [("dtype", _i32), ("group", _i32), ("rows", _i64), ("cols", _i64), ("eps", _dbl), ("x", _P),
                ("ld_x", _i64), ("residual", _P), ("ld_residual", _i64), ("weight", _P), ("h", _P), ("ld_h", _i64),
                ("y", _P), ("ld_y", _i64), ("q8", _P), ("ld_q8", _i64), ("scale", _P), ("rstd", _P)]


class RmsNormBackwardArgs(ctypes.Structure):
    """Mirror of zero_rms_norm_backward_args_t."""
    _fields_ = [("dtype", _i32), ("pad_", _i32), ("rows", _i64), ("cols", _i64), ("dy", _P), ("ld_dy", _i64),
                ("h", _P), ("ld_h", _i64), ("weight", _P), ("rstd", _P), ("dh", _P), ("ld_dh", _i64), ("dx", _P),
                ("ld_dx", _i64), ("dweight", _P), ("workspace", _P), ("workspace_floats", _i64)]


class RouteArgs(ctypes.Structure):
    """Mirror of zero_route_args_t."""
    _fields_ = [("dtype", _i32), ("score", _i32), ("rows", _i64), ("experts", _i32), ("k", _i32), ("groups", _i32),
                ("top_groups", _i32), ("group_top", _i32), ("renormalise", _i32), ("scale", _dbl), ("logits", _P),
                ("ld_logits", _i64), ("bias", _P), ("index", _P), ("weight", _P)]


class RouteOrderArgs(ctypes.Structure):
    """Mirror of zero_route_order_args_t."""
    _fields_ = [("index", _P), ("slots", _i64), ("experts", _i32), ("pad_", _i32), ("offsets", _P), ("order", _P),
                ("workspace", _P), ("workspace_ints", _i64)]


class RouteBackwardArgs(ctypes.Structure):
    """Mirror of zero_route_backward_args_t."""
    _fields_ = [("dtype", _i32), ("score", _i32), ("rows", _i64), ("experts", _i32), ("k", _i32),
                ("renormalise", _i32), ("pad_", _i32), ("scale", _dbl), ("logits", _P), ("ld_logits", _i64),
                ("bias", _P), ("index", _P), ("dweight", _P), ("dlogits", _P), ("ld_dlogits", _i64)]


class DistillArgs(ctypes.Structure):
    """Mirror of zero_distill_args_t."""
    _fields_ = [("dtype", _i32), ("teacher_dtype", _i32), ("rows", _i64), ("vocab", _i64), ("k", _i32),
                ("pad_", _i32), ("temperature", _dbl), ("soft", _dbl), ("hard", _dbl), ("grad_scale", _dbl),
                ("logits", _P), ("ld_logits", _i64), ("teacher_index", _P), ("teacher_logits", _P), ("labels", _P),
                ("row_weight", _P), ("loss", _P), ("stats", _P), ("dloss", _P), ("dlogits", _P), ("ld_dlogits", _i64)]


EXPORTS = ("zero_rms_norm", "zero_rms_norm_backward", "zero_rms_norm_workspace", "zero_route", "zero_route_order",
           "zero_route_workspace", "zero_route_backward", "zero_distill_step", "zero_distill_loss",
           "zero_distill_backward")
for _f in EXPORTS:
    getattr(_lib, _f).restype = ctypes.c_int
    getattr(_lib, _f).argtypes = [_P, _P]
_lib.zero_rms_norm_workspace.argtypes = [_i64, _i64, ctypes.POINTER(_i64)]
_lib.zero_route_workspace.argtypes = [_i64, _i32, ctypes.POINTER(_i64)]


def _matrix(t, dtypes, what, rows=None, cols=None):
    """(address, rows, cols, elements from row to row) of a device matrix; None gives no address."""
    if t is None:
        return None, rows, cols, cols
    if t.dtype not in dtypes:
        raise TypeError("%s: dtype %s not in %s" % (what, t.dtype, dtypes))
    if not t.is_cuda:
        raise TypeError("%s must be a device tensor" % what)
    if t.dim() != 2:
        if t.dim() < 1:
            raise ValueError("%s must have a dimension" % what)
        t = t.view(-1, t.shape[-1]) if t.numel() else t.reshape(0, t.shape[-1])
    n, c = t.shape
    if (rows is not None and n != rows) or (cols is not None and c != cols):
        raise ValueError("%s has shape [%d, %d], not [%s, %s]" % (what, n, c, rows, cols))
    step, one = t.stride()
    if one != 1 and c > 1 and n > 0:
        raise ValueError("%s: the last dimension must be contiguous" % what)
    return t.data_ptr(), n, c, step if n > 1 else c


def _vector(t, dtypes, what, numel):
    """The address of a contiguous device array of `numel` elements (None gives none)."""
    if t is not None and t.numel() != numel:
        raise ValueError("%s has %d elements, not %d" % (what, t.numel(), numel))
    return _addr(t, dtypes, what)


def _room(t, dtype, what):
    """(address, elements) of a workspace, which may be None."""
    return (None, 0) if t is None else (_addr(t, (dtype,), what), t.numel())


_F32, _I32 = (torch.float32,), (torch.int32,)


def _types(t, what):
    if t.dtype not in _TYPE:
        raise TypeError("%s: dtype %s not in %s" % (what, t.dtype, tuple(_TYPE)))
    return (t.dtype,)


def zero_rms_norm(x, weight, eps, residual=None, h=None, y=None, q8=None, scale=None, group=0, rstd=None,
                  stream=None):
    """h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h * rstd * weight, and with q8 and scale the
    rows y in e4m3 (torch.float8_e4m3fn or uint8 codes) with one fp32 scale for each `group` columns (0: a row).
    Each output is written where a tensor is given; y, q8 * scale and h are [rows, cols], rstd [rows],
    scale [rows, ceil(cols / group)].  h may be residual or x in place, and so may y."""
    dt = _types(x, "x")
    px, rows, cols, ld_x = _matrix(x, dt, "x")
    pr, _, _, ld_r = _matrix(residual, dt, "residual", rows, cols)
    ph, _, _, ld_h = _matrix(h, dt, "h", rows, cols)
    py, _, _, ld_y = _matrix(y, dt, "y", rows, cols)
    pq, _, _, ld_q = _matrix(q8, _Q8, "q8", rows, cols)
    groups = -(-cols // group) if group > 0 else 1
    args = RmsNormArgs(_TYPE[x.dtype], group, rows, cols, eps, px, ld_x, pr, ld_r, _vector(weight, dt, "weight", cols),
                       ph, ld_h, py, ld_y, pq, ld_q, _vector(scale, _F32, "scale", rows * groups),
                       _vector(rstd, _F32, "rstd", rows))
    _check(_lib.zero_rms_norm(ctypes.addressof(args), _stream(stream)))


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
    dt = _types(h, "h")
    ph, rows, cols, ld_h = _matrix(h, dt, "h")
    pdy, _, _, ld_dy = _matrix(dy, dt, "dy", rows, cols)
    pdh, _, _, ld_dh = _matrix(dh, dt, "dh", rows, cols)
    pdx, _, _, ld_dx = _matrix(dx, dt, "dx", rows, cols)
    pw, n = _room(workspace, torch.float32, "workspace")
    args = RmsNormBackwardArgs(_TYPE[h.dtype], 0, rows, cols, pdy, ld_dy, ph, ld_h,
                               _vector(weight, dt, "weight", cols), _vector(rstd, _F32, "rstd", rows), pdh, ld_dh,
                               pdx, ld_dx, _vector(dweight, dt, "dweight", cols), pw, n)
    _check(_lib.zero_rms_norm_backward(ctypes.addressof(args), _stream(stream)))


def zero_route(logits, index, weight, score="softmax", bias=None, groups=1, top_groups=1, group_top=1,
               renormalise=True, scale=1.0, stream=None):
    """The choice of k experts for each row of logits [tokens, experts]: index (int32) and weight (float32), both
    [tokens, k], in falling order of the keys.  score: "softmax" or "sigmoid"; bias [experts] float32 acts on the
    choice alone; groups > 1 keeps the top_groups groups of the largest sums of their group_top largest keys."""
    dt = _types(logits, "logits")
    pl, rows, experts, ld = _matrix(logits, dt, "logits")
    k = index.shape[-1]
    if score not in _SCORE:
        raise ValueError("score must be one of %s" % (tuple(_SCORE),))
    args = RouteArgs(_TYPE[logits.dtype], _SCORE[score], rows, experts, k, groups, top_groups, group_top,
                     bool(renormalise), scale, pl, ld, _vector(bias, _F32, "bias", experts),
                     _vector(index, _I32, "index", rows * k), _vector(weight, _F32, "weight", rows * k))
    _check(_lib.zero_route(ctypes.addressof(args), _stream(stream)))


def zero_route_workspace(slots, experts):
    """Ints of workspace that zero_route_order needs for these sizes (at most 1024 * (experts + 1))."""
    out = _i64()
    _check(_lib.zero_route_workspace(int(slots), int(experts), ctypes.byref(out)))
    return out.value


def zero_route_order(index, experts, offsets, order, workspace=None, stream=None):
    """The slots (flat positions in index, int32) by expert, then by slot: order[offsets[e]:offsets[e + 1]] are
    expert e's; slots without an expert are left out and order ends in as many -1.  offsets [experts + 1] and order
    [slots] are int32; workspace: int32, at least zero_route_workspace(slots, experts) elements."""
    n = index.numel()
    pw, room = _room(workspace, torch.int32, "workspace")
    args = RouteOrderArgs(_addr(index, _I32, "index"), n, experts, 0,
                          _vector(offsets, _I32, "offsets", experts + 1), _vector(order, _I32, "order", n), pw, room)
    _check(_lib.zero_route_order(ctypes.addressof(args), _stream(stream)))


def zero_route_backward(logits, index, dweight, dlogits, score="softmax", bias=None, renormalise=True, scale=1.0,
                        stream=None):
    """The gradient of zero_route's logits into dlogits [tokens, experts] (may be logits in place) from that of its
    weights, dweight [tokens, k] float32, and its index."""
    dt = _types(logits, "logits")
    pl, rows, experts, ld = _matrix(logits, dt, "logits")
    pd, _, _, ld_d = _matrix(dlogits, dt, "dlogits", rows, experts)
    k = index.shape[-1]
    if score not in _SCORE:
        raise ValueError("score must be one of %s" % (tuple(_SCORE),))
    args = RouteBackwardArgs(_TYPE[logits.dtype], _SCORE[score], rows, experts, k, bool(renormalise), 0, scale, pl,
                             ld, _vector(bias, _F32, "bias", experts), _vector(index, _I32, "index", rows * k),
                             _vector(dweight, _F32, "dweight", rows * k), pd, ld_d)
    _check(_lib.zero_route_backward(ctypes.addressof(args), _stream(stream)))


def _distill(fn, logits, teacher_index, teacher_logits, loss, stats, dlogits, dloss, labels, soft, hard, temperature,
             row_weight, grad_scale, stream):
    dt = _types(logits, "logits")
    pl, rows, vocab, ld = _matrix(logits, dt, "logits")
    pd, _, _, ld_d = _matrix(dlogits, dt, "dlogits", rows, vocab)
    k = 0 if teacher_index is None else teacher_index.shape[-1]
    teacher = ZERO_F32
    if k:
        teacher = _TYPE[_types(teacher_logits, "teacher_logits")[0]]
    args = DistillArgs(_TYPE[logits.dtype], teacher, rows, vocab, k, 0, temperature, soft, hard, grad_scale, pl, ld,
                       _vector(teacher_index, _I32, "teacher_index", rows * k),
                       _vector(teacher_logits, None, "teacher_logits", rows * k),
                       _vector(labels, _I32, "labels", rows), _vector(row_weight, _F32, "row_weight", rows),
                       _vector(loss, _F32, "loss", rows), _vector(stats, _F32, "stats", 3 * rows),
                       _vector(dloss, _F32, "dloss", rows), pd, ld_d)
    _check(fn(ctypes.addressof(args), _stream(stream)))


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
