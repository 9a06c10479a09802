"""Python binding of the operators of a token model's training step that include/division.h declares beside the codec: the
root-mean-square norm with an output in 8 bits, the log probabilities of given tokens, the norm and clipping of all gradients.

Argument marshalling only, as in binding.py: device tensors in, device tensors out, all arithmetic in the HIP library, on torch's
current stream or the one given.  Token vectors are the last dimension of a tensor, next to one another; the dimensions before it may
have any stride that lets them count as rows (slices of a wider tensor do).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from . import binding
from .binding import OPERATOR_DESCS, OPERATOR_ENTRIES, OPERATOR_OTHERS, DivisionError, _dt, _result, _stream, lib

_vp, _i64, _ci, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
_CODES = {None: 0, "int8": 1, "e4m3": 2}
_CODE_TYPES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


class _NormDesc(ctypes.Structure):
    """division_norm of include/division.h"""
    _fields_ = [("x", _vp), ("residual", _vp), ("weight", _vp), ("x_stride", _i64), ("residual_stride", _i64), ("T", _i64), ("D", _i64),
                ("dt", _ci), ("weight_dt", _ci), ("eps", ctypes.c_float), ("sum", _vp), ("y", _vp), ("rstd", _vp), ("code", _ci),
                ("group", _ci), ("codes", _vp), ("scales", _vp)]


class _NormBackDesc(ctypes.Structure):
    """division_norm_back of include/division.h"""
    _fields_ = [("grad_y", _vp), ("sum", _vp), ("grad_sum", _vp), ("weight", _vp), ("rstd", _vp), ("grad_y_stride", _i64), ("sum_stride", _i64),
                ("grad_sum_stride", _i64), ("T", _i64), ("D", _i64), ("dt", _ci), ("weight_dt", _ci), ("grad_x", _vp), ("grad_weight", _vp),
                ("workspace", _vp), ("workspace_bytes", _sz)]


class _LogitsDesc(ctypes.Structure):
    """division_logits of include/division.h"""
    _fields_ = [("logits", _vp), ("ids", _vp), ("stride", _i64), ("T", _i64), ("V", _i64), ("ignore_index", _i64), ("dt", _ci), ("top", _ci), ("logp", _vp),
                ("entropy", _vp), ("lse", _vp), ("top_logp", _vp), ("top_ids", _vp), ("workspace", _vp), ("workspace_bytes", _sz)]


class _LogitsBackDesc(ctypes.Structure):
    """division_logits_back of include/division.h"""
    _fields_ = [("logits", _vp), ("ids", _vp), ("lse", _vp), ("entropy", _vp), ("grad_logp", _vp), ("grad_entropy", _vp), ("stride", _i64), ("grad_stride", _i64),
                ("T", _i64), ("V", _i64), ("ignore_index", _i64), ("dt", _ci), ("grad_logits", _vp)]


class _GradientDesc(ctypes.Structure):
    """division_gradient of include/division.h"""
    _fields_ = [("grad", _vp), ("out", _vp), ("n", _i64), ("dt", _ci), ("out_dt", _ci)]


OPERATOR_ENTRIES += [
    ("division_rms_norm", [_vp, _vp], _ci),
    ("division_read_codes", [_vp, _vp, _i64, _i64, _ci, _ci, _ci, _vp, _vp], _ci),
    ("division_rms_norm_backward_workspace", [_i64, _i64], _sz),
    ("division_rms_norm_backward", [_vp, _vp], _ci),
    ("division_log_probs_workspace", [_i64, _i64, _ci], _sz),
    ("division_log_probs_low", [_vp, _vp, _vp], _ci),
    ("division_log_probs_backward_low", [_vp, _vp, _vp], _ci),
    ("division_grad_norm_workspace", [_i64, _vp], _sz),
    ("division_clip_grads", [_i64, _vp, ctypes.c_float, _ci, _vp, _vp, _sz, _vp], _ci),
]
# the same without lse_low
OPERATOR_OTHERS += [("division_log_probs", [_vp, _vp], _ci), ("division_log_probs_backward", [_vp, _vp], _ci)]
OPERATOR_DESCS += [_NormDesc, _NormBackDesc, _LogitsDesc, _LogitsBackDesc, _GradientDesc]


def _fast():
    """The native side of the binding: plain calls (contiguous tensors, nothing handed in) take the host 4 to 8 us there, 12 to 15 through what
    stands below, which serves every other one."""
    return binding._fast or binding._load_fast()


def _checked(rc: int, what: str):
    if rc:
        raise DivisionError(rc, what)


def _rows(t: torch.Tensor, what: str):
    """(rows, their stride, columns) of a device tensor whose last dimension is one row."""
    if not t.is_cuda or t.dim() == 0 or (t.stride(-1) != 1 and t.shape[-1] != 1):
        raise ValueError(f"{what} must be a device tensor whose last dimension is contiguous")
    D = t.shape[-1]
    n = t.numel() // D if D else 0
    if t.dim() == 1 or n <= 1:
        return n if t.dim() > 1 else 1, D, D
    stride, inner = 0, 1                  # of the rows, from the innermost dimension that has more than one
    for size, st in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if inner == 1:
            stride = st
        elif st != stride * inner:
            raise ValueError(f"{what}: its leading dimensions do not count as rows of one stride")
        inner *= size
    return n, stride, D


def _dense(t: torch.Tensor, what: str, dtype=None, shape=None, device=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must have shape {tuple(shape)}")
    _beside(t, device, what)


def _beside(t: torch.Tensor, device, what: str):
    if device is not None and t.device != device:
        raise ValueError(f"{what} lies on another device")


def _at(t) -> int | None:
    return None if t is None else t.data_ptr()


def _written(*tensors):
    """Tensors of the caller's that a call writes over: autograd compares versions before it uses what it saved."""
    torch.autograd.graph.increment_version([t for t in tensors if t is not None and not t.is_inference()])


def _workspace(nbytes: int, device, stream):
    """Memory for one call.  torch hands it out again when the call's tensors are gone: to the current stream's next call, behind this
    one, or, where the call runs on another stream, not before that stream has passed it."""
    ws = torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)
    if stream is not None:
        ws.record_stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device))
    return ws


def _group_count(D: int, group: int) -> int:
    return -(-D // group) if group else 1


class Normed(NamedTuple):
    """What division_rms_norm returns; None for what was not asked for."""
    y: torch.Tensor | None
    sum: torch.Tensor                   # the residual stream behind the addition (x itself where there was none)
    rstd: torch.Tensor
    codes: torch.Tensor | None          # int8, or float8_e4m3fn
    scales: torch.Tensor | None


def _check_code(code, group):
    if code not in _CODES:
        raise ValueError("code is None, 'int8' or 'e4m3'")
    if group not in (0, 32, 64, 128):
        raise ValueError("a scale is for 32, 64 or 128 columns, or the row (0)")


def division_rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, residual: torch.Tensor | None = None, code: str | None = None,
                      group: int = 0, want_y: bool = True, stream=None) -> Normed:
    """Root-mean-square norm over the last dimension, of x + residual where a residual is given.

    code 'int8' or 'e4m3' gives the output in 8 bits too, with a scale for each row (group 0) or for 32, 64 or 128 of its columns;
    want_y=False then leaves y out.  x and residual: float32 or bfloat16; weight: either."""
    _check_code(code, group)
    if stream is None:
        got = _fast().rms_norm(x, weight, eps, residual, _CODES[code], group, want_y)
        if got is not None:
            return Normed._make(_result(got, "division_rms_norm"))
    T, xs, D = _rows(x, "x")
    _dense(weight, "weight", shape=(D,), device=x.device)
    dt, wdt = _dt(x.dtype), _dt(weight.dtype)
    rs = 0
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype:
            raise ValueError("residual must have x's shape and type")
        _beside(residual, x.device, "residual")
        _, rs, _ = _rows(residual, "residual")
    if not want_y and code is None:
        raise ValueError("want_y=False leaves nothing to compute without a code")
    lead = x.shape[:-1]
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_y else None
    total = torch.empty(x.shape, dtype=x.dtype, device=x.device) if residual is not None else x
    rstd = torch.empty(lead, dtype=torch.float32, device=x.device)
    codes = scales = None
    if code is not None:
        codes = torch.empty(x.shape, dtype=_CODE_TYPES[code], device=x.device)
        scales = torch.empty((*lead, _group_count(D, group)), dtype=torch.float32, device=x.device)
    d = _NormDesc(x.data_ptr(), _at(residual), weight.data_ptr(), xs, rs, T, D, dt, wdt, eps, total.data_ptr() if residual is not None else None,
                  _at(y), rstd.data_ptr(), _CODES[code], group, _at(codes), _at(scales))
    _checked(lib().division_rms_norm(ctypes.byref(d), _stream(stream)), "division_rms_norm")
    return Normed(y, total, rstd, codes, scales)


def division_read_codes(codes: torch.Tensor, scales: torch.Tensor, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                        stream=None) -> torch.Tensor:
    """The values of division_rms_norm's codes; the last dimension of scales says how many columns have one: the row, or 128, 64 or 32."""
    if out is None and stream is None:
        got = _fast().read_codes(codes, scales, dtype)
        if got is not None:
            return _result(got, "division_read_codes")
    code = {torch.int8: "int8", torch.float8_e4m3fn: "e4m3"}.get(codes.dtype)
    if code is None or codes.dim() == 0:
        raise TypeError("codes are int8 or float8_e4m3fn")
    _dense(codes, "codes")
    _dense(scales, "scales", dtype=torch.float32, device=codes.device)
    D, lead = codes.shape[-1], tuple(codes.shape[:-1])
    fits = [g for g in (0, 32, 64, 128) if tuple(scales.shape) == (*lead, _group_count(D, g))]
    if not fits:
        raise ValueError("scales do not fit the codes")
    group = fits[0]                     # more than one scale a row: of one group size alone
    if out is None:
        out = torch.empty(codes.shape, dtype=dtype, device=codes.device)
    else:
        _dense(out, "out", shape=codes.shape, device=codes.device)
        _written(out)
    if D == 0:
        raise DivisionError(1, "division_read_codes")
    _checked(lib().division_read_codes(codes.data_ptr(), scales.data_ptr(), codes.numel() // D, D, _CODES[code], group, _dt(out.dtype),
                                       out.data_ptr(), _stream(stream)), "division_read_codes")
    return out


def division_rms_norm_backward(grad_y: torch.Tensor, sum: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor,
                               grad_sum: torch.Tensor | None = None, out: torch.Tensor | None = None, stream=None):
    """(the gradient of x, which is the residual's too, the gradient of weight) from the gradient of y and what the forward call gave.

    grad_sum: the gradient that the residual stream brings from further on.  out: where the gradient of x goes (grad_y, sum or grad_sum
    themselves, for instance)."""
    if out is None and stream is None:
        got = _fast().rms_norm_backward(grad_y, sum, weight, rstd, grad_sum)
        if got is not None:
            return _result(got, "division_rms_norm_backward")
    T, ss, D = _rows(sum, "sum")
    _dense(weight, "weight", shape=(D,), device=sum.device)
    _dense(rstd, "rstd", dtype=torch.float32, shape=sum.shape[:-1], device=sum.device)
    dt, wdt = _dt(sum.dtype), _dt(weight.dtype)
    strides = []
    for name, g in (("grad_y", grad_y), ("grad_sum", grad_sum)):
        if g is not None and (g.shape != sum.shape or g.dtype != sum.dtype):
            raise ValueError(f"{name} must have sum's shape and type")
        if g is not None:
            _beside(g, sum.device, name)
        strides.append(_rows(g, name)[1] if g is not None else 0)
    if out is None:
        out = torch.empty(sum.shape, dtype=sum.dtype, device=sum.device)
    else:
        _dense(out, "out", dtype=sum.dtype, shape=sum.shape, device=sum.device)
        _written(out)
    grad_weight = torch.empty_like(weight)
    nbytes = int(lib().division_rms_norm_backward_workspace(T, D))
    ws = _workspace(nbytes, sum.device, stream)
    d = _NormBackDesc(grad_y.data_ptr(), sum.data_ptr(), _at(grad_sum), weight.data_ptr(), rstd.data_ptr(), strides[0], ss, strides[1], T, D, dt, wdt,
                      out.data_ptr(), grad_weight.data_ptr(), ws.data_ptr(), nbytes)
    _checked(lib().division_rms_norm_backward(ctypes.byref(d), _stream(stream)), "division_rms_norm_backward")
    return out, grad_weight


class LogProbs(NamedTuple):
    """What division_log_probs returns; None for what was not asked for."""
    logp: torch.Tensor
    entropy: torch.Tensor | None
    lse: torch.Tensor
    top_logp: torch.Tensor | None
    top_ids: torch.Tensor | None


def division_log_probs(logits: torch.Tensor, ids: torch.Tensor, top: int = 0, want_entropy: bool = True, ignore_index: int = -100,
                       stream=None, lse_low: torch.Tensor | None = None) -> LogProbs:
    """Log probability of ids[...] among logits[..., V] (float32 or bfloat16), the entropy and, for top > 0, the `top` most probable tokens (at most 64).

    ids: int64.  Where it is ignore_index the log probability is 0; any other number outside the vocabulary gives NaN.  Logits of -inf are tokens
    that cannot be; a row of nothing else has log probability -inf and entropy 0.

    lse_low (float32, a number for each row) receives what lse's rounding left out, for the backward pass: without it the gradient's probabilities are
    off by lse's last bit, 3e-5 of themselves at an lse of 500."""
    if stream is None:
        got = _fast().log_probs(logits, ids, top, want_entropy, ignore_index, lse_low)
        if got is not None:
            return LogProbs._make(_result(got, "division_log_probs"))
    T, stride, V = _rows(logits, "logits")
    lead = logits.shape[:-1]
    _dense(ids, "ids", dtype=torch.int64, shape=lead, device=logits.device)
    dt = _dt(logits.dtype)
    if lse_low is not None:
        _dense(lse_low, "lse_low", dtype=torch.float32, shape=lead, device=logits.device)
    if not 0 <= top <= min(64, V):
        raise ValueError("top is 0 to 64, and at most the vocabulary")
    f32 = dict(dtype=torch.float32, device=logits.device)
    logp, lse = torch.empty(lead, **f32), torch.empty(lead, **f32)
    entropy = torch.empty(lead, **f32) if want_entropy else None
    top_logp = torch.empty((*lead, top), **f32) if top else None
    top_ids = torch.empty((*lead, top), dtype=torch.int64, device=logits.device) if top else None
    nbytes = int(lib().division_log_probs_workspace(T, V, top))
    ws = _workspace(nbytes, logits.device, stream) if nbytes else None
    d = _LogitsDesc(logits.data_ptr(), ids.data_ptr(), stride, T, V, ignore_index, dt, top, logp.data_ptr(), _at(entropy), lse.data_ptr(), _at(top_logp),
                    _at(top_ids), _at(ws), nbytes)
    _checked(lib().division_log_probs_low(ctypes.byref(d), _at(lse_low), _stream(stream)), "division_log_probs")
    _written(lse_low)
    return LogProbs(logp, entropy, lse, top_logp, top_ids)


def division_log_probs_backward(logits: torch.Tensor, ids: torch.Tensor, lse: torch.Tensor, grad_logp: torch.Tensor, entropy: torch.Tensor | None = None,
                                grad_entropy: torch.Tensor | None = None, ignore_index: int = -100, out: torch.Tensor | None = None,
                                stream=None, lse_low: torch.Tensor | None = None) -> torch.Tensor:
    """The gradient of logits from those of logp and of the entropy (None: no gradient comes that way).

    lse, entropy and lse_low (None: zeros) are what division_log_probs gave.  out: where the gradient goes; out=logits overwrites them, which saves a step its second-largest
    tensor."""
    if out is None and stream is None:
        got = _fast().log_probs_backward(logits, ids, lse, grad_logp, entropy, grad_entropy, ignore_index, lse_low)
        if got is not None:
            return _result(got, "division_log_probs_backward")
    T, stride, V = _rows(logits, "logits")
    lead = logits.shape[:-1]
    _dense(ids, "ids", dtype=torch.int64, shape=lead, device=logits.device)
    dt = _dt(logits.dtype)
    if grad_entropy is not None and entropy is None:
        raise ValueError("the entropy's gradient needs the entropy")
    for name, t in (("lse", lse), ("grad_logp", grad_logp), ("entropy", entropy), ("grad_entropy", grad_entropy), ("lse_low", lse_low)):
        if t is not None:
            _dense(t, name, dtype=torch.float32, shape=lead, device=logits.device)
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    elif out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out must have the logits' shape and type")
    else:
        _written(out)
    _beside(out, logits.device, "out")
    _, out_stride, _ = _rows(out, "out")
    d = _LogitsBackDesc(logits.data_ptr(), ids.data_ptr(), lse.data_ptr(), _at(entropy), grad_logp.data_ptr(), _at(grad_entropy), stride, out_stride, T, V,
                        ignore_index, dt, out.data_ptr())
    _checked(lib().division_log_probs_backward_low(ctypes.byref(d), _at(lse_low), _stream(stream)), "division_log_probs_backward")
    return out


def _fills_its_memory(t: torch.Tensor) -> bool:
    """Whether the elements lie next to one another in some order of the dimensions (channels-last weights do, for instance)."""
    if t.is_contiguous():
        return True
    expected = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != expected:
            return False
        expected *= size
    return True


def _grads(grads, out, limit, stream, what):
    if stream is None:
        got = _fast().clip_grads(grads, out, limit)
        if got is not None:
            return _result(got, what)
    grads = list(grads)
    outs = grads if out is None else list(out)
    if len(outs) != len(grads):
        raise ValueError("one output per gradient")
    if not grads:
        raise ValueError("no gradients")
    device = grads[0].device
    descs = (_GradientDesc * len(grads))()
    for i, (g, o) in enumerate(zip(grads, outs)):
        if not g.is_cuda or not _fills_its_memory(g):
            raise ValueError("every gradient must be a device tensor whose elements lie next to one another")
        _beside(g, device, "a gradient")
        if o is not g:
            # element by element in memory: the same order on both sides
            if o.shape != g.shape or not (o.is_contiguous() and g.is_contiguous() or o.stride() == g.stride()):
                raise ValueError("an output must have its gradient's shape and strides")
            _beside(o, device, "an output")
        n = g.numel()
        descs[i] = _GradientDesc(g.data_ptr() if n else None, o.data_ptr() if n else None, n, _dt(g.dtype), _dt(o.dtype))
    norm = torch.empty((), dtype=torch.float32, device=device)
    nbytes = int(lib().division_grad_norm_workspace(len(grads), descs))
    ws = _workspace(nbytes, device, stream)
    _checked(lib().division_clip_grads(len(grads), descs, limit if limit is not None else 0.0, limit is not None, norm.data_ptr(), ws.data_ptr(), nbytes,
                                       _stream(stream)), what)
    if limit is not None:
        _written(*outs)
    return norm


def division_grad_norm(grads, stream=None) -> torch.Tensor:
    """The 2-norm of all elements of a list of gradients (float32 or bfloat16, mixed as they come): one float32 on the device."""
    return _grads(grads, None, None, stream, "division_grad_norm")


def division_clip_grads(grads, max_norm: float, out=None, stream=None) -> torch.Tensor:
    """Scales the gradients by min(1, max_norm / (norm + 1e-6)), in place or into the tensors of `out` (of the same shapes and strides; float32
    outputs for bfloat16 gradients, for instance), and returns their norm before that.  Nothing waits for the device: where the
    norm is not finite the gradients are not either, and the caller that wants to skip the step looks at it."""
    if not max_norm >= 0:
        raise ValueError("max_norm is a number from 0 up")
    return _grads(grads, out, float(max_norm), stream, "division_clip_grads")
