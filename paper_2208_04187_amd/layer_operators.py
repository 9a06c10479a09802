"""Python binding of the operators of a token model's layers that include/division.h declares: attention with its backward pass, the norms of queries and
keys with the rotation by their positions, rows of the tokens' table with its gradient, dropout without a stored mask.

Argument marshalling only, as in operators.py: device tensors in, device tensors out, all arithmetic in the HIP library, on torch's current stream or the one given.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple

import torch

from .binding import LAYER_DESCS, LAYER_ENTRIES, _dt, _memory, _result, _stream, lib
from .operators import _at, _beside, _checked, _dense, _fast, _rows, _written

_vp, _i64, _ci, _sz, _f, _u64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t, ctypes.c_float, ctypes.c_uint64
_three, _two, _pair = _i64 * 3, _i64 * 2, _vp * 2


class _AttentionDesc(ctypes.Structure):
    """division_attention of include/division.h"""
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("q_strides", _three), ("k_strides", _three), ("v_strides", _three), ("B", _i64), ("Sq", _i64), ("Sk", _i64), ("H", _i64),
                ("G", _i64), ("D", _i64), ("dt", _ci), ("scale", _f), ("causal", _ci), ("window", _i64), ("lengths", _vp), ("starts", _vp)]


class _AttentionBackDesc(ctypes.Structure):
    """division_attention_back of include/division.h"""
    _fields_ = [("grad_out", _vp), ("out", _vp), ("lse", _vp), ("grad_out_strides", _three), ("grad_q", _vp), ("grad_k", _vp), ("grad_v", _vp), ("workspace", _vp),
                ("workspace_bytes", _sz)]


class _RotateDesc(ctypes.Structure):
    """division_rotate of include/division.h"""
    _fields_ = [("x", _pair), ("weight", _pair), ("token_strides", _two), ("head_strides", _two), ("heads", _two), ("weight_dt", _ci * 2), ("T", _i64), ("D", _i64), ("rotated", _i64),
                ("dt", _ci), ("next", _ci), ("eps", _f), ("frequencies", _vp), ("positions", _vp), ("y", _pair), ("rstd", _pair)]


class _RotateBackDesc(ctypes.Structure):
    """division_rotate_back of include/division.h"""
    _fields_ = [("grad_y", _pair), ("rstd", _pair), ("token_strides", _two), ("head_strides", _two), ("grad_x", _pair), ("grad_weight", _pair), ("workspace", _vp), ("workspace_bytes", _sz)]


class _EmbeddingBackDesc(ctypes.Structure):
    """division_embedding_back of include/division.h"""
    _fields_ = [("grad", _vp), ("ids", _vp), ("grad_stride", _i64), ("T", _i64), ("V", _i64), ("D", _i64), ("ignore_index", _i64), ("dt", _ci), ("table_dt", _ci), ("scale", _f),
                ("add", _ci), ("grad_table", _vp), ("workspace", _vp), ("workspace_bytes", _sz)]


LAYER_ENTRIES += [
    ("division_attention_workspace", [_vp], _sz),
    ("division_attend", [_vp, _vp, _vp, _vp, _sz, _vp], _ci),
    ("division_attention_backward_workspace", [_vp], _sz),
    ("division_attention_backward", [_vp, _vp, _vp], _ci),
    ("division_head_norm_rotate", [_vp, _vp], _ci),
    ("division_head_norm_rotate_backward_workspace", [_i64, _i64], _sz),
    ("division_head_norm_rotate_backward", [_vp, _vp, _vp], _ci),
    ("division_embedding", [_vp, _i64, _vp, _i64, _i64, _ci, _f, _i64, _vp, _vp], _ci),
    ("division_embedding_backward_workspace", [_i64, _i64, _i64], _sz),
    ("division_embedding_backward", [_vp, _vp], _ci),
    ("division_dropout_add", [_vp, _vp, _i64, _ci, ctypes.c_double, _u64, _vp, _vp, _vp], _ci),
]
LAYER_DESCS += [_AttentionDesc, _AttentionBackDesc, _RotateDesc, _RotateBackDesc, _EmbeddingBackDesc]


class _Call:
    """One call: its outputs and workspace on the device of its tensors, in the memory of its stream, and the launch there, whatever the current device."""

    def __init__(self, device, stream, what):
        self.device, self.stream, self.what = device, stream, what
        self.make = _memory(stream, device)

    def new(self, shape, dtype):
        return self.make(torch.empty, shape, dtype=dtype, device=self.device)

    def workspace(self, nbytes: int):
        return self.make(torch.empty, max(int(nbytes), 1), dtype=torch.uint8, device=self.device, given=False)

    def launch(self, entry, *args):
        if self.device.index == torch.cuda.current_device():
            _checked(entry(*args, _stream(self.stream)), self.what)
        else:
            with torch.cuda.device(self.device):
                _checked(entry(*args, _stream(self.stream)), self.what)


class Attended(NamedTuple):
    """What division_attention returns."""
    out: torch.Tensor                   # [batch, queries, heads, features]
    lse: torch.Tensor                   # float32 [batch, heads, queries]: ln of the sum of the scores' exponentials


def _heads(t: torch.Tensor, what: str, like: torch.Tensor | None = None):
    """Strides of a device tensor [batch, tokens, heads, features] whose features lie next to one another."""
    if not t.is_cuda or t.dim() != 4 or (t.stride(3) != 1 and t.shape[3] != 1):
        raise ValueError(f"{what} must be a device tensor [batch, tokens, heads, features] whose last dimension is contiguous")
    if like is not None:
        if t.dtype != like.dtype:
            raise TypeError(f"{what} must be {like.dtype}")
        _beside(t, like.device, what)
    return _three(*(0 if n == 1 else s for n, s in zip(t.shape[:3], t.stride()[:3])))


def _attention(q, k, v, scale, causal, window, lengths, starts):
    d = _AttentionDesc()
    d.q_strides, d.k_strides, d.v_strides = _heads(q, "q"), _heads(k, "k", q), _heads(v, "v", q)
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1], k.shape[2]
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        raise ValueError("k and v must have one shape, q's batch and features")
    if G == 0 or H % G:
        raise ValueError("the query heads must be a multiple of the key heads")
    for name, t in (("lengths", lengths), ("starts", starts)):
        if t is not None:
            _dense(t, name, dtype=torch.int32, shape=(B,), device=q.device)
    if not 0 <= window < 2 ** 63:
        raise ValueError("window is a whole number from 0 up")
    d.q, d.k, d.v = q.data_ptr(), k.data_ptr(), v.data_ptr()
    d.B, d.Sq, d.Sk, d.H, d.G, d.D, d.dt = B, Sq, Sk, H, G, D, _dt(q.dtype)
    d.scale = 1.0 / math.sqrt(D) if scale is None and D else scale or 0.0
    d.causal, d.window, d.lengths, d.starts = bool(causal), window, _at(lengths), _at(starts)
    return d


def division_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float | None = None, causal: bool = False, window: int = 0,
                       lengths: torch.Tensor | None = None, starts: torch.Tensor | None = None, stream=None) -> Attended:
    """softmax(scale q k^T) v over the keys that a query sees.

    q [batch, queries, heads, features], k and v [batch, keys, key heads, features], float32 or bfloat16; features a multiple of 8 up to 128, every row on 16 bytes (slices of a
    projection's output and of a cache are).  Query head h reads key head h // (heads / key heads).  scale: 1 / sqrt(features).

    lengths (int32 [batch]): keys that a sequence has; what lies behind them is not looked at.  starts (int32 [batch]): where a sequence's first query stands among the keys, keys -
    queries if not given.  causal: a query sees no key behind its own position; window: only keys nearer than that.  What no query of a sequence can see behind its last key
    or before its first one is not looked at either.  A query that sees none has out 0 and lse -inf."""
    if stream is None:
        got = _fast().attention(q, k, v, scale, causal, window, lengths, starts)
        if got is not None:
            return Attended._make(_result(got, "division_attention"))
    d = _attention(q, k, v, scale, causal, window, lengths, starts)
    call = _Call(q.device, stream, "division_attention")
    out, lse = call.new(q.shape, q.dtype), call.new((q.shape[0], q.shape[2], q.shape[1]), torch.float32)
    nbytes = int(lib().division_attention_workspace(ctypes.byref(d)))
    ws = call.workspace(nbytes) if nbytes else None
    call.launch(lib().division_attend, ctypes.byref(d), out.data_ptr(), lse.data_ptr(), _at(ws), nbytes)
    return Attended(out, lse)


def division_attention_backward(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, scale: float | None = None,
                                causal: bool = False, window: int = 0, lengths: torch.Tensor | None = None, starts: torch.Tensor | None = None, stream=None):
    """(the gradients of q, of k and of v) from that of out, and from what division_attention gave for the same arguments."""
    if stream is None:
        got = _fast().attention_backward(q, k, v, scale, causal, window, lengths, starts, grad_out, out, lse)
        if got is not None:
            return _result(got, "division_attention_backward")
    d = _attention(q, k, v, scale, causal, window, lengths, starts)
    b = _AttentionBackDesc()
    b.grad_out_strides = _heads(grad_out, "grad_out", q)
    if grad_out.shape != q.shape:
        raise ValueError("grad_out must have q's shape")
    _dense(out, "out", dtype=q.dtype, shape=q.shape, device=q.device)
    _dense(lse, "lse", dtype=torch.float32, shape=(q.shape[0], q.shape[2], q.shape[1]), device=q.device)
    call = _Call(q.device, stream, "division_attention_backward")
    dq, dk, dv = (call.new(t.shape, t.dtype) for t in (q, k, v))
    nbytes = int(lib().division_attention_backward_workspace(ctypes.byref(d)))
    ws = call.workspace(nbytes)
    b.grad_out, b.out, b.lse, b.grad_q, b.grad_k, b.grad_v = grad_out.data_ptr(), out.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr()
    b.workspace, b.workspace_bytes = ws.data_ptr(), nbytes
    call.launch(lib().division_attention_backward, ctypes.byref(d), ctypes.byref(b))
    return dq, dk, dv


_PAIRS = {"halves": False, "next": True}


class Rotated(NamedTuple):
    """What division_head_norm_rotate returns; None for keys that were not given."""
    q: torch.Tensor
    k: torch.Tensor | None
    q_rstd: torch.Tensor                # float32 [..., heads]
    k_rstd: torch.Tensor | None


def _tokens_of_heads(t: torch.Tensor, what: str):
    """(tokens, their stride, heads, their stride, features) of a device tensor [..., heads, features]"""
    if not t.is_cuda or t.dim() < 2 or (t.stride(-1) != 1 and t.shape[-1] != 1):
        raise ValueError(f"{what} must be a device tensor [..., heads, features] whose last dimension is contiguous")
    T, stride, _ = _rows(t[..., 0, :], what) if t.shape[-2] else (0, 0, 0)
    return T, stride, t.shape[-2], t.stride(-2) if t.shape[-2] > 1 else 0, t.shape[-1]


def _rotation(q, k, q_weight, k_weight, frequencies, positions, eps, pairs):
    if pairs not in _PAIRS:
        raise ValueError("pairs is 'halves' or 'next'")
    if (k is None) != (k_weight is None):
        raise ValueError("keys and their norm's weight come together")
    d = _RotateDesc()
    sides = [(q, q_weight, "q")] + ([(k, k_weight, "k")] if k is not None else [])
    lead = q.shape[:-2]
    for i, (x, w, name) in enumerate(sides):
        T, stride, heads, head_stride, D = _tokens_of_heads(x, name)
        if x.shape[:-2] != lead or D != q.shape[-1] or x.dtype != q.dtype:
            raise ValueError("k must have q's tokens, features and type")
        _beside(x, q.device, name)
        _dense(w, f"{name}_weight", shape=(D,), device=q.device)
        if heads == 0:
            raise ValueError(f"{name} has no heads")
        d.x[i], d.weight[i], d.weight_dt[i] = x.data_ptr(), w.data_ptr(), _dt(w.dtype)
        d.token_strides[i], d.head_strides[i], d.heads[i] = stride, head_stride, heads
        d.T, d.D = T, D
    _dense(frequencies, "frequencies", dtype=torch.float64, device=q.device)
    if frequencies.dim() != 1:
        raise ValueError("frequencies is one row")
    _dense(positions, "positions", dtype=torch.int64, shape=lead, device=q.device)
    d.rotated, d.dt, d.next, d.eps = 2 * frequencies.numel(), _dt(q.dtype), _PAIRS[pairs], eps
    d.frequencies, d.positions = _at(frequencies) if frequencies.numel() else None, positions.data_ptr()
    return d, [x for x, _, _ in sides]


def division_head_norm_rotate(q: torch.Tensor, k: torch.Tensor | None, q_weight: torch.Tensor, k_weight: torch.Tensor | None, frequencies: torch.Tensor, positions: torch.Tensor,
                              eps: float = 1e-6, pairs: str = "halves", stream=None) -> Rotated:
    """Root-mean-square norms of queries and keys, head by head, and their rotation by position, in one pass.

    q [..., heads, features] and k [..., key heads, features] (or None): float32 or bfloat16, features even and up to 512; parts of one projection's output are fine.
    The first 2 * len(frequencies) features are turned by positions[...] * frequencies (int64, float64; angles are taken in 64 bits): feature p with p + len(frequencies)
    (pairs='halves') or 2 p with 2 p + 1 ('next').  The weights ([features], float32 or bfloat16) are the norms'."""
    if stream is None and pairs in _PAIRS:
        got = _fast().head_norm_rotate(q, k, q_weight, k_weight, frequencies, positions, eps, _PAIRS[pairs])
        if got is not None:
            return Rotated._make(_result(got, "division_head_norm_rotate"))
    d, sides = _rotation(q, k, q_weight, k_weight, frequencies, positions, eps, pairs)
    call = _Call(q.device, stream, "division_head_norm_rotate")
    ys = [call.new(x.shape, x.dtype) for x in sides]
    rstds = [call.new(x.shape[:-1], torch.float32) for x in sides]
    for i, (y, r) in enumerate(zip(ys, rstds)):
        d.y[i], d.rstd[i] = y.data_ptr(), r.data_ptr()
    call.launch(lib().division_head_norm_rotate, ctypes.byref(d))
    return Rotated(ys[0], ys[1] if k is not None else None, rstds[0], rstds[1] if k is not None else None)


def division_head_norm_rotate_backward(grad_q: torch.Tensor, grad_k: torch.Tensor | None, q: torch.Tensor, k: torch.Tensor | None, q_weight: torch.Tensor,
                                       k_weight: torch.Tensor | None, frequencies: torch.Tensor, positions: torch.Tensor, q_rstd: torch.Tensor, k_rstd: torch.Tensor | None,
                                       pairs: str = "halves", stream=None):
    """(the gradients of q, k and of their weights) from those of division_head_norm_rotate's q and k, its inputs and its rstd; None for keys that are not given."""
    if stream is None and pairs in _PAIRS:
        got = _fast().head_norm_rotate_backward(q, k, q_weight, k_weight, frequencies, positions, 0.0, _PAIRS[pairs], grad_q, grad_k, q_rstd, k_rstd)
        if got is not None:
            return _result(got, "division_head_norm_rotate_backward")
    d, sides = _rotation(q, k, q_weight, k_weight, frequencies, positions, 0.0, pairs)
    if (k is None) != (grad_k is None) or (k is None) != (k_rstd is None):
        raise ValueError("keys, their gradient and their statistic come together")
    b = _RotateBackDesc()
    call = _Call(q.device, stream, "division_head_norm_rotate_backward")
    dxs = [call.new(x.shape, x.dtype) for x in sides]
    dws = [call.new(w.shape, w.dtype) for w in ((q_weight, k_weight) if k is not None else (q_weight,))]
    for i, (x, g, r, name) in enumerate(zip(sides, (grad_q, grad_k), (q_rstd, k_rstd), ("q", "k"))):
        if g.shape != x.shape or g.dtype != x.dtype:
            raise ValueError(f"grad_{name} must have {name}'s shape and type")
        _beside(g, x.device, f"grad_{name}")
        _, b.token_strides[i], _, b.head_strides[i], _ = _tokens_of_heads(g, f"grad_{name}")
        _dense(r, f"{name}_rstd", dtype=torch.float32, shape=x.shape[:-1], device=x.device)
        b.grad_y[i], b.rstd[i], b.grad_x[i], b.grad_weight[i] = g.data_ptr(), r.data_ptr(), dxs[i].data_ptr(), dws[i].data_ptr()
    nbytes = int(lib().division_head_norm_rotate_backward_workspace(d.T, d.D))
    ws = call.workspace(nbytes)
    b.workspace, b.workspace_bytes = ws.data_ptr(), nbytes
    call.launch(lib().division_head_norm_rotate_backward, ctypes.byref(d), ctypes.byref(b))
    return (dxs[0], dxs[1], dws[0], dws[1]) if k is not None else (dxs[0], None, dws[0], None)


def division_embedding(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0, ignore_index: int = -100, stream=None) -> torch.Tensor:
    """scale * table[ids]: ids int64 of any shape, table [vocabulary, features] float32 or bfloat16.  Where ids is ignore_index the row is zeros; any other number outside the
    vocabulary gives NaN."""
    if stream is None:
        got = _fast().embedding(ids, table, scale, ignore_index)
        if got is not None:
            return _result(got, "division_embedding")
    _dense(table, "table")
    if table.dim() != 2:
        raise ValueError("table is [vocabulary, features]")
    _dense(ids, "ids", dtype=torch.int64, device=table.device)
    V, D = table.shape
    call = _Call(table.device, stream, "division_embedding")
    dt = _dt(table.dtype)
    out = call.new((*ids.shape, D), table.dtype)
    call.launch(lib().division_embedding, ids.data_ptr(), ids.numel(), table.data_ptr(), V, D, dt, scale, ignore_index, out.data_ptr())
    return out


def division_embedding_backward(grad: torch.Tensor, ids: torch.Tensor, vocabulary: int, scale: float = 1.0, ignore_index: int = -100, out: torch.Tensor | None = None,
                                add: bool = False, stream=None) -> torch.Tensor:
    """The gradient of division_embedding's table, [vocabulary, features], from that of its rows: each row's tokens are added up in their order.

    out: where it goes (float32 for bfloat16 gradients, for instance); add=True adds to what out holds, and leaves rows without a token alone."""
    if stream is None and out is None and not add:
        got = _fast().embedding_backward(grad, ids, vocabulary, scale, ignore_index)
        if got is not None:
            return _result(got, "division_embedding_backward")
    T, stride, D = _rows(grad, "grad")
    _dense(ids, "ids", dtype=torch.int64, shape=grad.shape[:-1], device=grad.device)
    call = _Call(grad.device, stream, "division_embedding_backward")
    if out is None:
        if add:
            raise ValueError("add=True adds to out")
        out = call.new((vocabulary, D), grad.dtype)
    else:
        _dense(out, "out", shape=(vocabulary, D), device=grad.device)
    nbytes = int(lib().division_embedding_backward_workspace(T, vocabulary, D))
    ws = call.workspace(nbytes)
    d = _EmbeddingBackDesc(grad.data_ptr(), ids.data_ptr(), stride, T, vocabulary, D, ignore_index, _dt(grad.dtype), _dt(out.dtype), scale, bool(add), out.data_ptr(), ws.data_ptr(),
                           nbytes)
    call.launch(lib().division_embedding_backward, ctypes.byref(d))
    _written(out)
    return out


def division_dropout_add(x: torch.Tensor, p: float, seed, residual: torch.Tensor | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """residual + V (.) x / (1 - p), without a stored mask: V is division_dropout_forward's of the same p and seed, and computed again for the gradient, by the same call on it
    without a residual.

    x and residual: contiguous, float32 or bfloat16.  seed: a whole number, or an int64 tensor of one element on the device, which is read when the kernel runs (a captured
    graph drops other elements when it is replayed with another).  out may be x or residual itself."""
    if stream is None and out is None:
        got = _fast().dropout_add(x, p, seed, residual)
        if got is not None:
            return _result(got, "division_dropout_add")
    _dense(x, "x")
    if residual is not None:
        _dense(residual, "residual", dtype=x.dtype, shape=x.shape, device=x.device)
    at = None
    if isinstance(seed, torch.Tensor):
        _dense(seed, "seed", dtype=torch.int64, device=x.device)
        if seed.numel() != 1:
            raise ValueError("seed is one number")
        at, seed = seed.data_ptr(), 0
    call = _Call(x.device, stream, "division_dropout_add")
    if out is None:
        out = call.new(x.shape, x.dtype)
    else:
        _dense(out, "out", dtype=x.dtype, shape=x.shape, device=x.device)
        _written(out)
    n = x.numel()
    call.launch(lib().division_dropout_add, x.data_ptr() if n else None, _at(residual) if n else None, n, _dt(x.dtype), p, seed & (2 ** 64 - 1), at, out.data_ptr() if n else None)
    return out
