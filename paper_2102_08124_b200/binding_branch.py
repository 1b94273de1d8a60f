"""ctypes binding of the residual branch's operators (dropout from a counter-based generator, root-mean-square norm) and of the
verification of drafted tokens.  Same names as include/tm.h, tensors in, tensors out; argument marshalling only.

Matrices, streams and outputs as in binding_train.  Random numbers hang on (seed, offset) alone: another call that is to have other numbers gives
another seed or offset.  offset_dev (int64[1] on the device, or None) is added to the offset when the kernel runs, for calls in a captured graph."""
from __future__ import annotations

import ctypes
import functools

from . import binding
from . import binding_train as bt
from .binding import TmError
from .binding_train import TM_ERR_RANGE

TM_DRAFT_MAX = 1024

_ready = None
_torch = None


def _lib():
    global _ready, _torch
    if _ready is None:
        lib = bt._lib()
        vp, i32, i64, u64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
        f32, random = ctypes.c_float, [ctypes.c_double, u64, u64, vp]
        lib.tm_dropout.argtypes = [vp, i64, vp, i64, i32, i64, i64] + random + [vp, i64, vp]
        lib.tm_rms_norm.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i32, f32] + random + [vp, i64, vp, i64, vp, vp]
        lib.tm_rms_norm_e4m3.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i32, f32, i32, vp, i64, vp, i64, vp, vp, vp]
        lib.tm_rms_norm_workspace_bytes.argtypes = [i64, i64]; lib.tm_rms_norm_workspace_bytes.restype = sz
        lib.tm_rms_norm_backward.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, i64] + random + [vp, i64, vp, i64, vp, vp, sz, vp]
        lib.tm_verify_draft.argtypes = [vp, i32, i64, i64, i64, i64, vp, i64, vp, f32, f32, u64, u64, vp, vp, vp, vp, vp, vp]
        for f in (lib.tm_dropout, lib.tm_rms_norm, lib.tm_rms_norm_e4m3, lib.tm_rms_norm_backward, lib.tm_verify_draft):
            f.restype = i32
        _torch = bt._torch
        _ready = lib
    return _ready


def _whole(seed, offset):
    """Both as they are: ctypes would cut them to 64 bits without a word."""
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise TmError(TM_ERR_RANGE, "seed and offset must be whole numbers from 0 to 2^64 - 1")


def _weight(weight, cols, device, default):
    kind = default if weight is None else weight.dtype
    code = 1 if kind is _torch.bfloat16 else 0 if kind is _torch.float32 else -1
    if code < 0:
        raise TmError(5, "weight must be float32 or bfloat16")
    return kind, code, bt._array(weight, (cols,), kind, device, "weight")


def _offset(offset_dev, device):
    return None if offset_dev is None else bt._array(offset_dev, (1,), _torch.int64, device, "offset_dev")


def tm_dropout(x, p: float, seed: int, offset: int = 0, residual=None, y=None, offset_dev=None, stream=None):
    """Dropout of x, plus residual where given.  The gradient of x is tm_dropout(dy, p, seed, offset); nothing is stored."""
    if stream is not None:
        return binding._under(stream, tm_dropout, locals())
    lib = _lib()
    code, dev, rows, cols, ld = bt._input(x, "x")
    _whole(seed, offset)
    ld_r = ld_y = cols
    if residual is not None:
        ld_r = bt._other(residual, "residual", x)
    if y is not None:
        ld_y = bt._other(y, "y", x)
    else:
        y = bt._like(x)
    bt._call(lib.tm_dropout, dev, x.data_ptr(), ld, bt._ptr(residual), ld_r, code, rows, cols, p, seed, offset, _offset(offset_dev, dev), y.data_ptr(), ld_y)
    return y


def tm_rms_norm(x, weight=None, eps: float = 1e-5, residual=None, p: float = 0.0, seed: int = 0, offset: int = 0, offset_dev=None, y=None,
                sum_out=None, rstd_out=None, want_sum: bool = True, want_stats: bool = True, stream=None):
    """Root-mean-square norm of dropout(x) (+ residual) over the columns.  Returns (y, the sum, rstd); the sum is None where it would be x
    itself (no residual, p = 0), unless sum_out was passed in."""
    if stream is not None:
        return binding._under(stream, tm_rms_norm, locals())
    lib = _lib()
    code, dev, rows, cols, ld = bt._input(x, "x")
    _, wcode, wp = _weight(weight, cols, dev, x.dtype)
    _whole(seed, offset)
    ld_r = ld_s = ld_y = cols
    if residual is not None:
        ld_r = bt._other(residual, "residual", x)
    if sum_out is not None:
        ld_s = bt._other(sum_out, "sum_out", x)
    elif want_sum and (residual is not None or p > 0):
        sum_out = bt._like(x)
    if y is not None:
        ld_y = bt._other(y, "y", x)
    else:
        y = bt._like(x)
    rp = None
    if rstd_out is not None:
        rp = bt._array(rstd_out, (rows,), _torch.float32, dev, "rstd_out")
    elif want_stats:
        rstd_out = _torch.empty(rows, dtype=_torch.float32, device=dev)
        rp = rstd_out.data_ptr()
    bt._call(lib.tm_rms_norm, dev, x.data_ptr(), ld, bt._ptr(residual), ld_r, code, rows, cols, wp, wcode, eps, p, seed, offset, _offset(offset_dev, dev),
             bt._ptr(sum_out), ld_s, y.data_ptr(), ld_y, rp)
    if cols == 0 and rstd_out is not None:                  # of which the entry writes nothing
        rstd_out.fill_(float("nan"))
    return y, sum_out, rstd_out


def tm_rms_norm_e4m3(x, weight=None, eps: float = 1e-5, residual=None, group: int = 0, y8=None, scales_out=None, sum_out=None, rstd_out=None,
                     want_sum: bool = True, stream=None):
    """The norm of x (+ residual) in 8 bits.  Returns (y8 float8_e4m3fn [rows, cols], scales float32 [rows, groups], the sum or None): y is
    y8 times its group's scale, a group being `group` columns (32, 64 or 128), or the row (0)."""
    if stream is not None:
        return binding._under(stream, tm_rms_norm_e4m3, locals())
    lib = _lib()
    code, dev, rows, cols, ld = bt._input(x, "x")
    _, wcode, wp = _weight(weight, cols, dev, x.dtype)
    if group not in (0, 32, 64, 128):
        raise TmError(TM_ERR_RANGE, binding.tm_status_string(TM_ERR_RANGE))
    ld_r = ld_s = ld_y = cols
    if residual is not None:
        ld_r = bt._other(residual, "residual", x)
    if sum_out is not None:
        ld_s = bt._other(sum_out, "sum_out", x)
    elif want_sum and residual is not None:
        sum_out = bt._like(x)
    e4m3, f32 = _torch.float8_e4m3fn, _torch.float32
    if y8 is None:
        y8 = _torch.empty_like(x, dtype=e4m3) if x.is_contiguous() else _torch.empty(rows, cols, dtype=e4m3, device=dev)
    else:
        if y8.dtype is not e4m3:
            raise TmError(5, "y8 must be float8_e4m3fn")
        if y8.shape != x.shape or y8.device != dev or (cols > 1 and y8.stride(1) != 1 and rows > 0):
            raise TmError(2, "y8 must have the shape and device of x, and unit column stride")
        ld_y = y8.stride(0) if rows > 1 else cols
    groups = -(-cols // group) if group else 1
    if scales_out is None:
        scales_out = _torch.empty(rows, groups, dtype=f32, device=dev)
        sp = scales_out.data_ptr()
    else:
        sp = bt._array(scales_out, (rows, groups), f32, dev, "scales_out")
    bt._call(lib.tm_rms_norm_e4m3, dev, x.data_ptr(), ld, bt._ptr(residual), ld_r, code, rows, cols, wp, wcode, eps, group, bt._ptr(sum_out), ld_s,
             y8.data_ptr(), ld_y, sp, bt._array(rstd_out, (rows,), f32, dev, "rstd_out"))
    if cols == 0:                                           # of which the entry writes nothing
        for t in (scales_out, rstd_out):
            if t is not None:
                t.fill_(float("nan"))
    return y8, scales_out, sum_out


@functools.lru_cache(maxsize=64)
def _workspace_bytes(rows, cols):
    return _lib().tm_rms_norm_workspace_bytes(rows, cols)


def tm_rms_norm_workspace_bytes(rows: int, cols: int) -> int:
    return _lib().tm_rms_norm_workspace_bytes(rows, cols)


def tm_rms_norm_backward(dy, h, rstd, weight=None, dsum=None, p: float = 0.0, seed: int = 0, offset: int = 0, offset_dev=None, dh=None, dx=None,
                         dweight_out=None, workspace=None, want_dh: bool = True, want_weight: bool = True, params_dtype=None, stream=None):
    """Gradients of the norm of h (x, or the sum that tm_rms_norm returned).  Returns (dh, dx, dweight): dh the gradient of the sum and of the
    residual (None with want_dh=False where p > 0), dx that of x (dh itself with p = 0, unless dx was passed in), dweight of the weight's dtype (without
    a weight `params_dtype`, or h's; None with want_weight=False)."""
    if stream is not None:
        return binding._under(stream, tm_rms_norm_backward, locals())
    lib = _lib()
    code, dev, rows, cols, ld_h = bt._input(h, "h")
    kind, wcode, wp = _weight(weight, cols, dev, params_dtype or h.dtype)
    _whole(seed, offset)
    ld_dy, ld_s, ld_dh, ld_dx = bt._other(dy, "dy", h), cols, cols, cols
    if dsum is not None:
        ld_s = bt._other(dsum, "dsum", h)
    if dh is not None:
        ld_dh = bt._other(dh, "dh", h)
    elif want_dh or (p == 0 and dx is None):
        dh = bt._like(h)
    if dx is not None:
        ld_dx = bt._other(dx, "dx", h)
    elif p != 0:
        dx = bt._like(h)
    wsp, bytes_, dwp = None, 0, None
    if dweight_out is not None:
        dwp = bt._array(dweight_out, (cols,), kind, dev, "dweight_out")
    elif want_weight:
        dweight_out = _torch.empty(cols, dtype=kind, device=dev)
        dwp = dweight_out.data_ptr()
    if dwp is not None:
        if workspace is None:
            bytes_ = _workspace_bytes(rows, cols)
            workspace = _torch.empty(bytes_, dtype=_torch.uint8, device=dev)
        else:
            if workspace.device != dev or not workspace.is_contiguous():
                raise TmError(8, "workspace must be a contiguous tensor on the matrix's device")
            bytes_ = workspace.numel() * workspace.element_size()
        wsp = workspace.data_ptr()
    bt._call(lib.tm_rms_norm_backward, dev, dy.data_ptr(), ld_dy, h.data_ptr(), ld_h, code, rows, cols, wp, wcode,
             bt._array(rstd, (rows,), _torch.float32, dev, "rstd"), bt._ptr(dsum), ld_s, p, seed, offset, _offset(offset_dev, dev), bt._ptr(dh), ld_dh,
             bt._ptr(dx), ld_dx, dwp, wsp, bytes_)
    return dh, dh if dx is None else dx, dweight_out


def tm_verify_draft(logits, draft_logits, draft_ids, seed: int, offset: int = 0, temperature: float = 1.0, draft_temperature=None, offset_dev=None,
                    tokens_out=None, accepted_out=None, logp_out=None, want_logp: bool = True, status=None, stream=None):
    """Drafted tokens against the target's probabilities.  logits [batch * (drafted + 1), vocab], draft_logits [batch * drafted, vocab] (None: a
    drafter that was certain), draft_ids int32 [batch, drafted], negative behind a sequence's last draft; draft_temperature: None for `temperature`.
    Returns (tokens int32 [batch, drafted + 1], accepted int32 [batch], log-probabilities float32 [batch, drafted + 1] or None).
    status: int32[1] or None.  With drafted = 0 it draws a token from every row of logits."""
    if stream is not None:
        return binding._under(stream, tm_verify_draft, locals())
    lib = _lib()
    code, dev, rows, vocab, ld = bt._input(logits, "logits")
    if draft_ids.dim() != 2:
        raise TmError(2, "draft_ids must be [batch, drafted]")
    batch, drafted = draft_ids.shape
    i32, f32, shape, ld_d = _torch.int32, _torch.float32, (batch, drafted + 1), vocab
    if rows != batch * (drafted + 1) or drafted > TM_DRAFT_MAX:
        raise TmError(2, "logits must have batch * (drafted + 1) rows, drafted being at most %d" % TM_DRAFT_MAX)
    _whole(seed, offset)
    if draft_logits is not None:
        if draft_logits.shape != (batch * drafted, vocab) or draft_logits.dtype is not logits.dtype or draft_logits.device != dev:
            raise TmError(2, "draft_logits must be [batch * drafted, vocab], of the dtype and device of logits")
        if vocab > 1 and drafted and batch and draft_logits.stride(1) != 1:
            raise TmError(2, "draft_logits must have unit column stride")
        ld_d = draft_logits.stride(0) if batch * drafted > 1 else vocab
    empty, lp = _torch.empty, None
    if tokens_out is None:
        tokens_out = empty(batch, drafted + 1, dtype=i32, device=dev)
        tp = tokens_out.data_ptr()
    else:
        tp = bt._array(tokens_out, shape, i32, dev, "tokens_out")
    if accepted_out is None:
        accepted_out = empty(batch, dtype=i32, device=dev)
        ap = accepted_out.data_ptr()
    else:
        ap = bt._array(accepted_out, (batch,), i32, dev, "accepted_out")
    if logp_out is not None:
        lp = bt._array(logp_out, shape, f32, dev, "logp_out")
    elif want_logp:
        logp_out = empty(batch, drafted + 1, dtype=f32, device=dev)
        lp = logp_out.data_ptr()
    bt._call(lib.tm_verify_draft, dev, logits.data_ptr(), code, batch, drafted, vocab, ld, bt._ptr(draft_logits), ld_d,
             bt._array(draft_ids, (batch, drafted), i32, dev, "draft_ids"), temperature, temperature if draft_temperature is None else draft_temperature,
             seed, offset, _offset(offset_dev, dev), tp, ap, lp, bt._array(status, (1,), i32, dev, "status"))
    return tokens_out, accepted_out, logp_out
