"""ctypes binding of the operators of the training step around the masked layers: layer norm with a residual sum, a teacher's
largest logits, and the distillation loss against such lists.  Same names as include/tm.h, tensors in, tensors out; argument
marshalling only.

Matrices are 2-D CUDA tensors, float32 or bfloat16, with unit column stride; rows may be strided.  Every call is asynchronous on
`stream` (a torch.cuda.Stream) or torch's current stream, and creates whichever outputs were not passed in."""
from __future__ import annotations

import ctypes

from . import binding
from .binding import TmError

TM_DEV_BADID = 8
TM_ERR_RANGE = 11
TM_TOP_MAX = 256

_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = binding.load_library()
        vp, i32, i64, sz, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        lib.tm_layer_norm.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, vp, i32, f32, vp, i64, vp, i64, vp, vp, vp]
        lib.tm_layer_norm_workspace_bytes.argtypes = [i64, i64]; lib.tm_layer_norm_workspace_bytes.restype = sz
        lib.tm_layer_norm_backward.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        lib.tm_top_logits.argtypes = [vp, i32, i64, i64, i64, i32, f32, vp, vp, vp, vp, vp]
        lists = [vp, i32, i64, i64, i64, vp, vp, i32, vp, vp, f32, f32]
        lib.tm_distill_loss.argtypes = lists + [vp, vp, vp, vp]
        lib.tm_distill_grad.argtypes = lists + [vp, vp, vp, i64, vp, vp]
        lib.tm_distill_loss_grad.argtypes = lists + [vp, vp, i64, vp, vp]
        for f in (lib.tm_layer_norm, lib.tm_layer_norm_backward, lib.tm_top_logits, lib.tm_distill_loss, lib.tm_distill_grad, lib.tm_distill_loss_grad):
            f.restype = i32
        _ready = lib
    return _ready


def _call(fn, device, stream, *args):
    """fn(*args, stream) with `device` current."""
    import torch
    s = (stream if stream is not None else torch.cuda.current_stream(device)).cuda_stream
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, s)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, s)
    if rc != 0:
        raise TmError(rc, binding.tm_status_string(rc))


def _matrix(t, what, like=None):
    """Checks a 2-D matrix (of the shape, type and device of `like`); returns its leading dimension."""
    if t.dim() != 2 or not t.is_cuda or (t.shape[1] > 1 and t.stride(1) != 1):
        raise TmError(2, "%s must be a 2-D CUDA tensor with unit column stride" % what)
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise TmError(2, "%s must have the shape, dtype and device of the input matrix" % what)
    rows, cols = t.shape
    return t.stride(0) if rows > 1 else cols


def _array(t, shape, dtype, device, what):
    """Checks a small contiguous array; returns its address, or None for None."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TmError(5, "%s must be %s" % (what, dtype))
    if tuple(t.shape) != shape or t.device != device or not t.is_contiguous():
        raise TmError(2, "%s must be a contiguous tensor of shape %s on the matrix's device" % (what, shape))
    return t.data_ptr()


def _params(weight, bias, cols, device, default):
    import torch
    kind = weight.dtype if weight is not None else bias.dtype if bias is not None else default
    code = 0 if kind == torch.float32 else 1 if kind == torch.bfloat16 else None
    if code is None:
        raise TmError(5, "weight and bias must be float32 or bfloat16")
    return kind, code, _array(weight, (cols,), kind, device, "weight"), _array(bias, (cols,), kind, device, "bias")


def _code(t, what):
    import torch
    if t.dtype == torch.bfloat16:
        return 1
    if t.dtype == torch.float32:
        return 0
    raise TmError(5, "%s must be float32 or bfloat16" % what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def tm_layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None, y=None, sum_out=None, mean_out=None, rstd_out=None,
                  want_sum: bool = True, want_stats: bool = True, stream=None):
    """Layer norm of x, or of x + residual, over the columns.  Returns (y, x + residual or None, mean, rstd)."""
    import torch
    dev = x.device
    code, ld = _code(x, "x"), _matrix(x, "x")
    rows, cols = x.shape
    _, wcode, wp, bp = _params(weight, bias, cols, dev, x.dtype)
    ld_r = _matrix(residual, "residual", x) if residual is not None else cols
    if residual is None:
        sum_out = None
    elif sum_out is None and want_sum:
        sum_out = torch.empty((rows, cols), dtype=x.dtype, device=dev)
    if y is None:
        y = torch.empty((rows, cols), dtype=x.dtype, device=dev)
    if want_stats:
        if mean_out is None:
            mean_out = torch.empty((rows,), dtype=torch.float32, device=dev)
        if rstd_out is None:
            rstd_out = torch.empty((rows,), dtype=torch.float32, device=dev)
    ld_s = _matrix(sum_out, "sum_out", x) if sum_out is not None else cols
    _call(_lib().tm_layer_norm, dev, stream, x.data_ptr(), ld, _ptr(residual), ld_r, code, rows, cols, wp, bp, wcode, eps, _ptr(sum_out), ld_s,
          y.data_ptr(), _matrix(y, "y", x), _array(mean_out, (rows,), torch.float32, dev, "mean_out"), _array(rstd_out, (rows,), torch.float32, dev, "rstd_out"))
    return y, sum_out, mean_out, rstd_out


def tm_layer_norm_workspace_bytes(rows: int, cols: int) -> int:
    return int(_lib().tm_layer_norm_workspace_bytes(rows, cols))


def tm_layer_norm_backward(dy, h, mean, rstd, weight=None, dsum=None, dx=None, dweight_out=None, dbias_out=None, workspace=None,
                           want_params: bool = True, params_dtype=None, stream=None):
    """Gradients of the layer norm of h (x, or the sum that tm_layer_norm returned).  Returns (dx, dweight, dbias); the last two have
    the weight's dtype (without a weight `params_dtype`, or h's), and are None with want_params=False."""
    import torch
    dev = h.device
    code, ld_h = _code(h, "h"), _matrix(h, "h")
    rows, cols = h.shape
    kind, wcode, wp, _ = _params(weight, None, cols, dev, params_dtype or h.dtype)
    if dx is None:
        dx = torch.empty((rows, cols), dtype=h.dtype, device=dev)
    bytes_ = 0
    if want_params:
        if dweight_out is None:
            dweight_out = torch.empty((cols,), dtype=kind, device=dev)
        if dbias_out is None:
            dbias_out = torch.empty((cols,), dtype=kind, device=dev)
    if dweight_out is not None or dbias_out is not None:
        if workspace is None:
            workspace = torch.empty((tm_layer_norm_workspace_bytes(rows, cols),), dtype=torch.uint8, device=dev)
        bytes_ = workspace.numel() * workspace.element_size()
    _call(_lib().tm_layer_norm_backward, dev, stream, dy.data_ptr(), _matrix(dy, "dy", h), h.data_ptr(), ld_h, code, rows, cols, wp, wcode,
          _array(mean, (rows,), torch.float32, dev, "mean"), _array(rstd, (rows,), torch.float32, dev, "rstd"),
          _ptr(dsum), _matrix(dsum, "dsum", h) if dsum is not None else cols, dx.data_ptr(), _matrix(dx, "dx", h),
          _array(dweight_out, (cols,), kind, dev, "dweight_out"), _array(dbias_out, (cols,), kind, dev, "dbias_out"), _ptr(workspace), bytes_)
    return dx, dweight_out, dbias_out


def tm_top_logits(logits, k: int, temperature: float = 1.0, values_out=None, ids_out=None, lse_out=None, want_lse: bool = True,
                  status=None, stream=None):
    """The k largest logits of every row (equal ones by the lower id) and log sum exp(logits / temperature).
    Returns (values float32 [rows, k], ids int32 [rows, k], lse float32 [rows] or None).  status: int32[1] or None."""
    import torch
    dev = logits.device
    code, ld = _code(logits, "logits"), _matrix(logits, "logits")
    rows, vocab = logits.shape
    if values_out is None:
        values_out = torch.empty((rows, max(k, 0)), dtype=torch.float32, device=dev)
    if ids_out is None:
        ids_out = torch.empty((rows, max(k, 0)), dtype=torch.int32, device=dev)
    if lse_out is None and want_lse:
        lse_out = torch.empty((rows,), dtype=torch.float32, device=dev)
    _call(_lib().tm_top_logits, dev, stream, logits.data_ptr(), code, rows, vocab, ld, k, temperature,
          _array(values_out, (rows, k), torch.float32, dev, "values_out"), _array(ids_out, (rows, k), torch.int32, dev, "ids_out"),
          _array(lse_out, (rows,), torch.float32, dev, "lse_out"), _array(status, (1,), torch.int32, dev, "status"))
    return values_out, ids_out, lse_out


def _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale):
    import torch
    dev = logits.device
    code, ld = _code(logits, "logits"), _matrix(logits, "logits")
    rows, vocab = logits.shape
    if top_ids.dim() != 2:
        raise TmError(2, "top_ids must be [rows, k]")
    k = top_ids.shape[1]
    return dev, rows, vocab, (logits.data_ptr(), code, rows, vocab, ld, _array(top_values, (rows, k), torch.float32, dev, "top_values"),
                              _array(top_ids, (rows, k), torch.int32, dev, "top_ids"), k, _array(teacher_lse, (rows,), torch.float32, dev, "teacher_lse"),
                              _array(row_weight, (rows,), torch.float32, dev, "row_weight"), temperature, scale)


def tm_distill_loss(logits, top_values, top_ids, teacher_lse=None, row_weight=None, temperature: float = 1.0, scale: float = 1.0,
                    loss_out=None, stats_out=None, want_stats: bool = True, status=None, stream=None):
    """Loss of every row (float32 [rows]) and the statistics [rows, 2] that tm_distill_grad takes."""
    import torch
    dev, rows, _, head = _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale)
    if loss_out is None:
        loss_out = torch.empty((rows,), dtype=torch.float32, device=dev)
    if stats_out is None and want_stats:
        stats_out = torch.empty((rows, 2), dtype=torch.float32, device=dev)
    _call(_lib().tm_distill_loss, dev, stream, *head, _array(loss_out, (rows,), torch.float32, dev, "loss_out"),
          _array(stats_out, (rows, 2), torch.float32, dev, "stats_out"), _array(status, (1,), torch.int32, dev, "status"))
    return loss_out, stats_out


def tm_distill_grad(logits, top_values, top_ids, stats, grad_loss=None, teacher_lse=None, row_weight=None, temperature: float = 1.0,
                    scale: float = 1.0, dlogits=None, status=None, stream=None):
    """Gradient of the logits from the statistics of tm_distill_loss, times grad_loss[row] where given."""
    import torch
    dev, rows, vocab, head = _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale)
    if dlogits is None:
        dlogits = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
    _call(_lib().tm_distill_grad, dev, stream, *head, _array(stats, (rows, 2), torch.float32, dev, "stats"),
          _array(grad_loss, (rows,), torch.float32, dev, "grad_loss"), dlogits.data_ptr(), _matrix(dlogits, "dlogits", logits),
          _array(status, (1,), torch.int32, dev, "status"))
    return dlogits


def tm_distill_loss_grad(logits, top_values, top_ids, teacher_lse=None, row_weight=None, temperature: float = 1.0, scale: float = 1.0,
                         loss_out=None, dlogits=None, status=None, stream=None):
    """Loss of every row and the gradient of their sum, in one pass over the logits.  Returns (loss [rows], dlogits)."""
    import torch
    dev, rows, vocab, head = _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale)
    if loss_out is None:
        loss_out = torch.empty((rows,), dtype=torch.float32, device=dev)
    if dlogits is None:
        dlogits = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
    _call(_lib().tm_distill_loss_grad, dev, stream, *head, _array(loss_out, (rows,), torch.float32, dev, "loss_out"),
          dlogits.data_ptr(), _matrix(dlogits, "dlogits", logits), _array(status, (1,), torch.int32, dev, "status"))
    return loss_out, dlogits
