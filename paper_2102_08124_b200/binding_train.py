"""ctypes binding of the operators of the training step around the masked layers: layer norm with a residual sum, a teacher's
largest logits, and the distillation loss against such lists.  Same names as include/tm.h, tensors in, tensors out; argument
marshalling only.

Matrices are 2-D CUDA tensors, float32 or bfloat16, with unit column stride; rows may be strided.  Every call is asynchronous on
`stream` (a torch.cuda.Stream) or torch's current stream, and creates whichever outputs were not passed in (on that stream: another one
that uses them has to wait for it)."""
from __future__ import annotations

import ctypes

from . import binding
from .binding import TmError

TM_DEV_BADID = 8
TM_ERR_RANGE = 11
TM_TOP_MAX = 256

_ready = None
_torch = None              # torch, once a call needed it: importing this package alone does not import torch
_raw_stream = None
_current_device = None


def _lib():
    global _ready, _torch, _raw_stream, _current_device
    if _ready is None:
        import torch
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
        _torch = torch
        # the address of the current stream without a Stream object around it (2 us less a call), where this torch has it
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _ready = lib
    return _ready


def _call(fn, device, *args):
    """fn(*args, torch's current stream) with `device` current."""
    index = device.index
    s = _raw_stream(index)
    if _current_device() == index:
        rc = fn(*args, s)
    else:
        with _torch.cuda.device(device):
            rc = fn(*args, s)
    if rc != 0:
        raise TmError(rc, binding.tm_status_string(rc))


def _input(t, what):
    """Checks the matrix of a call; returns its type's code, device, shape and leading dimension."""
    code = 1 if t.dtype is _torch.bfloat16 else 0 if t.dtype is _torch.float32 else -1
    if code < 0:
        raise TmError(5, "%s must be float32 or bfloat16" % what)
    if not t.is_cuda or t.dim() != 2:
        raise TmError(2, "%s must be a 2-D CUDA tensor" % what)
    rows, cols = t.shape
    step = t.stride()
    if cols > 1 and step[1] != 1 and rows > 0:
        raise TmError(2, "%s must have unit column stride" % what)
    return code, t.device, rows, cols, step[0] if rows > 1 else cols


def _other(t, what, like):
    """Checks a matrix of the shape, type and device of `like`; returns its leading dimension."""
    if t.shape != like.shape or t.dtype is not like.dtype or t.device != like.device:
        raise TmError(2, "%s must have the shape, dtype and device of the input matrix" % what)
    rows, cols = t.shape
    step = t.stride()
    if cols > 1 and step[1] != 1 and rows > 0:
        raise TmError(2, "%s must have unit column stride" % what)
    return step[0] if rows > 1 else cols


def _array(t, shape, dtype, device, what):
    """Checks a small contiguous array; returns its address, or None for None."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise TmError(5, "%s must be %s" % (what, dtype))
    if t.shape != shape or t.device != device or not t.is_contiguous():
        raise TmError(2, "%s must be a contiguous tensor of shape %s on the matrix's device" % (what, shape))
    return t.data_ptr()


def _params(weight, bias, cols, device, default):
    kind = weight.dtype if weight is not None else bias.dtype if bias is not None else default
    code = 1 if kind is _torch.bfloat16 else 0 if kind is _torch.float32 else -1
    if code < 0:
        raise TmError(5, "weight and bias must be float32 or bfloat16")
    return kind, code, _array(weight, (cols,), kind, device, "weight"), _array(bias, (cols,), kind, device, "bias")


def _like(t):
    """An output matrix: the shape of `t`, rows side by side."""
    return _torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _ptr(t):
    return None if t is None else t.data_ptr()


def tm_layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None, y=None, sum_out=None, mean_out=None, rstd_out=None,
                  want_sum: bool = True, want_stats: bool = True, stream=None):
    """Layer norm of x, or of x + residual, over the columns.  Returns (y, the sum, mean, rstd); the sum is None without a residual,
    unless sum_out was passed in (it receives x then)."""
    if stream is not None:
        return binding._under(stream, tm_layer_norm, locals())
    lib = _lib()
    code, dev, rows, cols, ld = _input(x, "x")
    _, wcode, wp, bp = _params(weight, bias, cols, dev, x.dtype)
    ld_r = ld_s = ld_y = cols
    if residual is not None:
        ld_r = _other(residual, "residual", x)
    if sum_out is not None:
        ld_s = _other(sum_out, "sum_out", x)
    elif residual is not None and want_sum:
        sum_out = _like(x)
    if y is not None:
        ld_y = _other(y, "y", x)
    else:
        y = _like(x)
    mp = rp = None
    f32 = _torch.float32
    if want_stats and mean_out is None and rstd_out is None:
        mean_out, rstd_out = _torch.empty((2, rows), dtype=f32, device=dev).unbind(0)
        mp, rp = mean_out.data_ptr(), rstd_out.data_ptr()
    else:
        if want_stats:
            mean_out = _torch.empty((rows,), dtype=f32, device=dev) if mean_out is None else mean_out
            rstd_out = _torch.empty((rows,), dtype=f32, device=dev) if rstd_out is None else rstd_out
        mp, rp = _array(mean_out, (rows,), f32, dev, "mean_out"), _array(rstd_out, (rows,), f32, dev, "rstd_out")
    _call(lib.tm_layer_norm, dev, x.data_ptr(), ld, _ptr(residual), ld_r, code, rows, cols, wp, bp, wcode, eps, _ptr(sum_out), ld_s,
          y.data_ptr(), ld_y, mp, rp)
    if cols == 0:                                           # of which the entry writes nothing
        for t in (mean_out, rstd_out):
            if t is not None:
                t.fill_(float("nan"))
    return y, sum_out, mean_out, rstd_out


def tm_layer_norm_workspace_bytes(rows: int, cols: int) -> int:
    return _lib().tm_layer_norm_workspace_bytes(rows, cols)


def tm_layer_norm_backward(dy, h, mean, rstd, weight=None, dsum=None, dx=None, dweight_out=None, dbias_out=None, workspace=None,
                           want_params: bool = True, params_dtype=None, stream=None):
    """Gradients of the layer norm of h (x, or the sum that tm_layer_norm returned).  Returns (dx, dweight, dbias); the last two have
    the weight's dtype (without a weight `params_dtype`, or h's), and are None with want_params=False."""
    if stream is not None:
        return binding._under(stream, tm_layer_norm_backward, locals())
    lib = _lib()
    code, dev, rows, cols, ld_h = _input(h, "h")
    kind, wcode, wp, _ = _params(weight, None, cols, dev, params_dtype or h.dtype)
    ld_dy, ld_s, ld_dx, f32 = _other(dy, "dy", h), cols, cols, _torch.float32
    if dsum is not None:
        ld_s = _other(dsum, "dsum", h)
    if dx is not None:
        ld_dx = _other(dx, "dx", h)
    else:
        dx = _like(h)
    wsp, bytes_, dwp, dbp = None, 0, None, None
    if want_params and dweight_out is None and dbias_out is None:
        dweight_out, dbias_out = _torch.empty((2, cols), dtype=kind, device=dev).unbind(0)
        dwp, dbp = dweight_out.data_ptr(), dbias_out.data_ptr()
    else:
        if want_params:
            dweight_out = _torch.empty((cols,), dtype=kind, device=dev) if dweight_out is None else dweight_out
            dbias_out = _torch.empty((cols,), dtype=kind, device=dev) if dbias_out is None else dbias_out
        dwp, dbp = _array(dweight_out, (cols,), kind, dev, "dweight_out"), _array(dbias_out, (cols,), kind, dev, "dbias_out")
    if dweight_out is not None or dbias_out is not None:
        if workspace is None:
            bytes_ = lib.tm_layer_norm_workspace_bytes(rows, cols)
            workspace = _torch.empty((bytes_,), dtype=_torch.uint8, device=dev)
        else:
            if workspace.device != dev or not workspace.is_contiguous():
                raise TmError(8, "workspace must be a contiguous tensor on the matrix's device")
            bytes_ = workspace.numel() * workspace.element_size()
        wsp = workspace.data_ptr()
    _call(lib.tm_layer_norm_backward, dev, dy.data_ptr(), ld_dy, h.data_ptr(), ld_h, code, rows, cols, wp, wcode,
          _array(mean, (rows,), f32, dev, "mean"), _array(rstd, (rows,), f32, dev, "rstd"), _ptr(dsum), ld_s, dx.data_ptr(), ld_dx, dwp, dbp, wsp, bytes_)
    return dx, dweight_out, dbias_out


def tm_top_logits(logits, k: int, temperature: float = 1.0, values_out=None, ids_out=None, lse_out=None, want_lse: bool = True,
                  status=None, stream=None):
    """The k largest logits of every row (equal ones by the lower id) and log sum exp(logits / temperature).
    Returns (values float32 [rows, k], ids int32 [rows, k], lse float32 [rows] or None).  status: int32[1] or None."""
    if stream is not None:
        return binding._under(stream, tm_top_logits, locals())
    lib = _lib()
    code, dev, rows, vocab, ld = _input(logits, "logits")
    if not 1 <= k <= TM_TOP_MAX:                            # before anything of that size is created
        raise TmError(TM_ERR_RANGE, binding.tm_status_string(TM_ERR_RANGE))
    f32, i32, shape = _torch.float32, _torch.int32, (rows, k)
    if values_out is None:
        values_out = _torch.empty(shape, dtype=f32, device=dev)
    if ids_out is None:
        ids_out = _torch.empty(shape, dtype=i32, device=dev)
    if lse_out is None and want_lse:
        lse_out = _torch.empty((rows,), dtype=f32, device=dev)
    _call(lib.tm_top_logits, dev, logits.data_ptr(), code, rows, vocab, ld, k, temperature, _array(values_out, shape, f32, dev, "values_out"),
          _array(ids_out, shape, i32, dev, "ids_out"), _array(lse_out, (rows,), f32, dev, "lse_out"), _array(status, (1,), i32, dev, "status"))
    return values_out, ids_out, lse_out


def _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale):
    code, dev, rows, vocab, ld = _input(logits, "logits")
    if top_ids.dim() != 2:
        raise TmError(2, "top_ids must be [rows, k]")
    k, f32 = top_ids.shape[1], _torch.float32
    return dev, rows, (logits.data_ptr(), code, rows, vocab, ld, _array(top_values, (rows, k), f32, dev, "top_values"),
                       _array(top_ids, (rows, k), _torch.int32, dev, "top_ids"), k, _array(teacher_lse, (rows,), f32, dev, "teacher_lse"),
                       _array(row_weight, (rows,), f32, dev, "row_weight"), temperature, scale)


def tm_distill_loss(logits, top_values, top_ids, teacher_lse=None, row_weight=None, temperature: float = 1.0, scale: float = 1.0,
                    loss_out=None, stats_out=None, want_stats: bool = True, status=None, stream=None):
    """Loss of every row (float32 [rows]) and the statistics [rows, 2] that tm_distill_grad takes."""
    if stream is not None:
        return binding._under(stream, tm_distill_loss, locals())
    lib = _lib()
    dev, rows, head = _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale)
    f32 = _torch.float32
    if loss_out is None:
        loss_out = _torch.empty((rows,), dtype=f32, device=dev)
    if stats_out is None and want_stats:
        stats_out = _torch.empty((rows, 2), dtype=f32, device=dev)
    _call(lib.tm_distill_loss, dev, *head, _array(loss_out, (rows,), f32, dev, "loss_out"),
          _array(stats_out, (rows, 2), f32, dev, "stats_out"), _array(status, (1,), _torch.int32, dev, "status"))
    return loss_out, stats_out


def tm_distill_grad(logits, top_values, top_ids, stats, grad_loss=None, teacher_lse=None, row_weight=None, temperature: float = 1.0,
                    scale: float = 1.0, dlogits=None, status=None, stream=None):
    """Gradient of the logits from the statistics of tm_distill_loss, times grad_loss[row] where given."""
    if stream is not None:
        return binding._under(stream, tm_distill_grad, locals())
    lib = _lib()
    dev, rows, head = _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale)
    f32, ld_d = _torch.float32, logits.shape[1]
    if dlogits is not None:
        ld_d = _other(dlogits, "dlogits", logits)
    else:
        dlogits = _like(logits)
    _call(lib.tm_distill_grad, dev, *head, _array(stats, (rows, 2), f32, dev, "stats"), _array(grad_loss, (rows,), f32, dev, "grad_loss"),
          dlogits.data_ptr(), ld_d, _array(status, (1,), _torch.int32, dev, "status"))
    return dlogits


def tm_distill_loss_grad(logits, top_values, top_ids, teacher_lse=None, row_weight=None, temperature: float = 1.0, scale: float = 1.0,
                         loss_out=None, dlogits=None, status=None, stream=None):
    """Loss of every row and the gradient of their sum, in one pass over the logits.  Returns (loss [rows], dlogits)."""
    if stream is not None:
        return binding._under(stream, tm_distill_loss_grad, locals())
    lib = _lib()
    dev, rows, head = _lists(logits, top_values, top_ids, teacher_lse, row_weight, temperature, scale)
    ld_d = logits.shape[1]
    if loss_out is None:
        loss_out = _torch.empty((rows,), dtype=_torch.float32, device=dev)
    if dlogits is not None:
        ld_d = _other(dlogits, "dlogits", logits)
    else:
        dlogits = _like(logits)
    _call(lib.tm_distill_loss_grad, dev, *head, _array(loss_out, (rows,), _torch.float32, dev, "loss_out"), dlogits.data_ptr(), ld_d,
          _array(status, (1,), _torch.int32, dev, "status"))
    return loss_out, dlogits
