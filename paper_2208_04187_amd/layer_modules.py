"""The operators of layer_operators.py under torch.autograd.

division_token_attention computes its probabilities again for the backward pass from the queries, the keys and one number a row.  Scores of rebuilt queries and keys would not belong to that number, so inside
division_saved_tensors all that it caches stays exact: it is saved as matrices, which the hook keeps.  Queries, keys and values that are parts of one projection's output are cached as
that output, once.

DivisionHeadNormRotation caches the tensors before the norm, as DivisionRMSNorm does: compressed under the hook where they are maps of their own (tokens x features).

DivisionEmbedding caches the tokens, DivisionResidualDropout nothing but its seed.

First derivatives only: a second one raises.  Only calls the binding.

A backward pass that is captured into a graph needs parameters that no eager graph still holds (drop its outputs first): torch adds a parameter's gradient up on the stream on which the first
graph met it, which a capture cannot leave.  The first call of a DivisionHeadNormRotation on a device copies its frequencies there: make it before the capture.
"""
from __future__ import annotations

import torch

from .autograd import _call_seed
from .layer_operators import (_tokens_of_heads, division_attention, division_attention_backward, division_dropout_add, division_embedding, division_embedding_backward,
                              division_head_norm_rotate, division_head_norm_rotate_backward)
from .token_modules import _beside_the_stream, _first_derivatives


def _fits(t: torch.Tensor) -> bool:
    """Whether attention takes the rows as they lie: on 16 bytes, features next to one another, tokens at most 8 MB apart and heads all within 1 GB"""
    if t.dim() != 4:
        return True                                         # for the call itself to refuse
    size = t.element_size()
    if t.data_ptr() % 16 or t.stride(3) != 1 or any(n > 1 and s * size % 16 for n, s in zip(t.shape[:3], t.stride()[:3])):
        return False
    return (t.shape[1] <= 1 or t.stride(1) * size <= 1 << 23) and (t.shape[2] <= 1 or t.stride(2) * size * t.shape[2] <= 1 << 30)


def _as_rows(t: torch.Tensor) -> torch.Tensor:
    """t, or a dense copy where attention does not take its rows as they lie (a dense tensor may begin off 16 bytes itself)"""
    return t if _fits(t) else t.clone(memory_format=torch.contiguous_format)


def _matrix(t: torch.Tensor) -> torch.Tensor:
    """[batch, tokens, heads, features] as [batch * tokens, heads * features], without a copy where the strides allow it"""
    return t.detach().reshape(t.shape[0] * t.shape[1], t.shape[2] * t.shape[3])


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, causal, window, lengths, starts):
        q, k, v = _as_rows(q), _as_rows(k), _as_rows(v)
        a = division_attention(q, k, v, scale, causal, window, lengths, starts)
        ctx.save_for_backward(*(_matrix(t) for t in (q, k, v, a.out)), a.lse.view(-1), lengths, starts)
        ctx.shapes, ctx.settings = (q.shape, k.shape), (scale, causal, window)
        ctx.mark_non_differentiable(a.lse)
        ctx.set_materialize_grads(False)
        return a.out, a.lse

    @staticmethod
    @_first_derivatives
    def backward(ctx, grad_out, grad_lse=None):
        if grad_out is None:
            return (None,) * 8
        q, k, v, out, lse, lengths, starts = ctx.saved_tensors
        of_q, of_k = ctx.shapes
        q, k, v, out = q.view(of_q), k.view(of_k), v.view(of_k), out.view(of_q)
        grads = division_attention_backward(_as_rows(grad_out), q, k, v, out, lse.view(of_q[0], of_q[2], of_q[1]), *ctx.settings, lengths, starts)
        return (*grads, None, None, None, None, None)


def division_token_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float | None = None, causal: bool = False, window: int = 0,
                             lengths: torch.Tensor | None = None, starts: torch.Tensor | None = None) -> torch.Tensor:
    """division_attention's out, with gradients for q, k and v."""
    return _Attention.apply(q, k, v, scale, bool(causal), int(window), lengths, starts)[0]


def _as_tokens(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy where its leading dimensions do not count as tokens of one stride"""
    try:
        _tokens_of_heads(t, "x")
    except ValueError:
        return t.contiguous() if t.is_cuda else t
    return t


class _Rotation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, frequencies, positions, eps, pairs):
        q, k = _as_tokens(q), _as_tokens(k)
        r = division_head_norm_rotate(q, k, q_weight, k_weight, frequencies, positions, eps, pairs)
        ctx.save_for_backward(q.detach().flatten(-2), k.detach().flatten(-2), q_weight, k_weight, frequencies, positions, r.q_rstd.view(-1), r.k_rstd.view(-1))
        ctx.shapes, ctx.pairs = (q.shape, k.shape), pairs
        ctx.set_materialize_grads(False)
        return r.q, r.k

    @staticmethod
    @_first_derivatives
    def backward(ctx, grad_q, grad_k):
        if grad_q is None and grad_k is None:
            return (None,) * 8
        q, k, q_weight, k_weight, frequencies, positions, q_rstd, k_rstd = ctx.saved_tensors
        q, k = (t.view(s) for t, s in zip((q, k), ctx.shapes))
        q_rstd, k_rstd = (t.view(s[:-1]) for t, s in zip((q_rstd, k_rstd), ctx.shapes))
        if grad_k is None:                              # only the queries were used
            dq, _, dwq, _ = division_head_norm_rotate_backward(grad_q.contiguous(), None, q, None, q_weight, None, frequencies, positions, q_rstd, None, ctx.pairs)
            return dq, None, dwq, None, None, None, None, None
        if grad_q is None:
            dk, _, dwk, _ = division_head_norm_rotate_backward(grad_k.contiguous(), None, k, None, k_weight, None, frequencies, positions, k_rstd, None, ctx.pairs)
            return None, dk, None, dwk, None, None, None, None
        dq, dk, dwq, dwk = division_head_norm_rotate_backward(grad_q.contiguous(), grad_k.contiguous(), q, k, q_weight, k_weight, frequencies, positions, q_rstd, k_rstd, ctx.pairs)
        return dq, dk, dwq, dwk, None, None, None, None


class DivisionHeadNormRotation(torch.nn.Module):
    """forward(q, k, positions) -> (q, k): root-mean-square norms of [..., heads, features] head by head, the first `rotated` features (all of them) turned by the token's position.

    positions: int64 of q's and k's leading dimensions."""

    def __init__(self, features: int, rotated: int | None = None, base: float = 10000.0, pairs: str = "halves", eps: float = 1e-6, device=None, dtype=None):
        super().__init__()
        rotated = features if rotated is None else int(rotated)
        if pairs not in ("halves", "next"):
            raise ValueError("pairs is 'halves' or 'next'")
        if features % 2 or rotated % 2 or not 0 <= rotated <= features:
            raise ValueError("features and rotated are even, and rotated at most features")
        self.eps, self.pairs, self.base, self.rotated = float(eps), pairs, float(base), rotated
        self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype)) for _ in range(2))
        self._frequencies = None

    def frequencies(self, device):
        # no buffer: a module's .to(dtype) would round it
        if self._frequencies is None or self._frequencies.device != device:
            with torch.inference_mode(False):               # kept for later calls, whose backward pass cannot take what was made in inference mode
                self._frequencies = torch.tensor([self.base ** (-p / self.rotated) for p in range(0, self.rotated, 2)], dtype=torch.float64).to(device)
        return self._frequencies

    def forward(self, q, k, positions):
        return _Rotation.apply(q, k, self.q_weight, self.k_weight, self.frequencies(q.device), positions.contiguous(), self.eps, self.pairs)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale, ignore_index):
        ctx.save_for_backward(ids)
        ctx.settings = (table.shape[0], scale, ignore_index)
        return division_embedding(ids, table, scale, ignore_index)

    @staticmethod
    @_first_derivatives
    def backward(ctx, grad):
        (ids,) = ctx.saved_tensors
        return None, division_embedding_backward(grad.contiguous(), ids, *ctx.settings), None, None


class DivisionEmbedding(torch.nn.Module):
    """forward(ids) -> scale * weight[ids], zeros where ids is ignore_index; the weight's gradient is added up in the order of the tokens."""

    def __init__(self, vocabulary: int, features: int, scale: float = 1.0, ignore_index: int = -100, device=None, dtype=None):
        super().__init__()
        self.scale, self.ignore_index = float(scale), int(ignore_index)
        self.weight = torch.nn.Parameter(torch.randn(vocabulary, features, device=device, dtype=dtype))

    def forward(self, ids):
        return _Embedding.apply(ids.contiguous(), self.weight, self.scale, self.ignore_index)


class _ResidualDropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed):
        ctx.settings, ctx.added = (p, seed), residual is not None
        return division_dropout_add(x.contiguous(), p, seed, residual=None if residual is None else residual.contiguous())

    @staticmethod
    @_first_derivatives
    def backward(ctx, grad):
        return division_dropout_add(grad.contiguous(), *ctx.settings) if ctx.needs_input_grad[0] else None, grad if ctx.added else None, None, None


class DivisionResidualDropout(torch.nn.Module):
    """forward(x, residual=None) -> residual + dropout(x), kept elements divided by 1 - p, without a stored mask.  Call number n of this module while training drops what seed + n says
    (DivisionDropout's elements of the same call): modules of a model need seeds farther apart than they have calls.  In eval mode nothing is dropped.  Under activation checkpointing seed is None: a call draws its own from torch's generator, which is put back before
    the forward runs again; a numbered call inside a backward pass raises.  A captured graph drops the captured call's elements whenever it is replayed: for others each time call
    division_dropout_add with a seed on the device."""

    def __init__(self, p: float = 0.5, seed: int | None = 0):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError("p is a probability")
        self.p, self.seed, self.calls = float(p), None if seed is None else int(seed), 0

    def forward(self, x, residual=None):
        x, residual = _beside_the_stream(x, residual)
        if not self.training or self.p == 0.0:
            return x if residual is None else x + residual
        return _ResidualDropout.apply(x, residual, self.p, _call_seed(self))
