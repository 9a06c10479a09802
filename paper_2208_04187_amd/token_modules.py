"""The operators of operators.py under torch.autograd: what a token model's training step does beside its products, with 8-bit or
compressed tensors cached for the backward pass.

DivisionRMSNorm caches the residual stream's sum and one number a row.  Inside division_saved_tensors the sum is cached compressed as any other
map of N x C x L (tokens x features) is.  All numbers that belong to rows (the norm's statistic, the codes' scales, lse and entropy) stay exact there: they are saved as
vectors and matrices, which the hook keeps, whatever dimensions the rows have.

DivisionNormLinear is a norm and the linear layer behind it.  The layer multiplies the norm's output in the model's own type; for its weight's gradient the
output is cached in 8 bits (int8 or e4m3, a scale for each row or for 32, 64 or 128 columns), the output itself is not kept.  Under autocast the layer's products are of its type, the norm of
the stream's.

division_token_log_probs is the loss: log probabilities and entropies with their gradients, alternatives beside them.  Of [tokens, vocabulary] only the logits are kept, and
`overwrite` hands their memory to their gradient.

First derivatives only: a second one raises.  Only calls the binding and torch's products.
"""
from __future__ import annotations

import functools

import torch
import torch.nn.functional as F

from .operators import (LogProbs, division_log_probs, division_log_probs_backward, division_read_codes, division_rms_norm,
                        division_rms_norm_backward)


class _NoSecond(torch.autograd.Function):
    """t, as the result of a graph that cannot be followed"""

    @staticmethod
    def forward(ctx, t, anchor):
        return t.view_as(t)

    @staticmethod
    def backward(ctx, grad):
        raise RuntimeError("trying to differentiate twice a function that has first derivatives only")


def _first_derivatives(backward):
    """Where a graph of the backward pass is asked for (create_graph), its results raise when they are differentiated.  (once_differentiable lets those through whose
    incoming gradient is a constant, as of out.sum(): a gradient penalty beside a loss would be dropped in silence.)"""
    @functools.wraps(backward)
    def first(ctx, *grads):
        with torch.no_grad():
            got = backward(ctx, *grads)
        if not torch.is_grad_enabled():
            return got
        anchor = torch.empty(0, requires_grad=True)
        return tuple(g if g is None else _NoSecond.apply(g, anchor) for g in got)
    return first


class _RMSNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        n = division_rms_norm(x, weight, eps, residual=residual)
        ctx.save_for_backward(n.sum, weight, n.rstd.view(-1))
        ctx.added = residual is not None
        ctx.set_materialize_grads(False)
        return (n.y, n.sum) if ctx.added else n.y

    @staticmethod
    @_first_derivatives
    def backward(ctx, grad_y, grad_sum=None):
        total, weight, rstd = ctx.saved_tensors
        if grad_y is None:                       # only the sum was used
            return grad_sum, grad_sum if ctx.added else None, None, None
        dx, dw = division_rms_norm_backward(grad_y.contiguous(), total, weight, rstd.view(total.shape[:-1]),
                                            grad_sum=None if grad_sum is None else grad_sum.contiguous())
        return dx, dx if ctx.added else None, dw, None


class _NormLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, norm_weight, weight, bias, eps, code, group):
        n = division_rms_norm(x, norm_weight, eps, residual=residual, code=code, group=group)
        ctx.save_for_backward(n.sum, norm_weight, n.rstd.view(-1), n.codes, n.scales.view(-1, n.scales.shape[-1]), weight)
        ctx.added, ctx.with_bias = residual is not None, bias is not None
        ctx.set_materialize_grads(False)
        out = F.linear(n.y, weight, bias)
        return (out, n.sum) if ctx.added else out

    @staticmethod
    @_first_derivatives
    def backward(ctx, grad_out, grad_sum=None):
        total, norm_weight, rstd, codes, scales, weight = ctx.saved_tensors
        if grad_out is None:
            return grad_sum, grad_sum if ctx.added else None, None, None, None, None, None, None
        # the products in the type of the forward pass's, which autocast may have chosen; gradients in their tensors' types
        g = grad_out.reshape(-1, grad_out.shape[-1])
        values = division_read_codes(codes.view(-1, codes.shape[-1]), scales, torch.bfloat16 if g.dtype == torch.bfloat16 else torch.float32).to(g.dtype)
        grad_weight = (g.t() @ values).to(weight.dtype) if ctx.needs_input_grad[3] else None
        grad_bias = g.sum(0).to(weight.dtype) if ctx.with_bias and ctx.needs_input_grad[4] else None
        grad_y = (g @ weight.to(g.dtype)).to(total.dtype).view(total.shape)
        dx, dw = division_rms_norm_backward(grad_y, total, norm_weight, rstd.view(total.shape[:-1]),
                                            grad_sum=None if grad_sum is None else grad_sum.contiguous())
        return dx, dx if ctx.added else None, dw, grad_weight, grad_bias, None, None, None


def _beside_the_stream(x, residual):
    """Under autocast a layer's output may be narrower than the stream it is added to: both in the wider type, as torch's own addition has it"""
    if residual is None or x.dtype == residual.dtype or not torch.is_autocast_enabled(x.device.type):
        return x, residual
    wide = torch.promote_types(x.dtype, residual.dtype)
    return x.to(wide), residual.to(wide)


class DivisionRMSNorm(torch.nn.Module):
    """forward(x, residual=None) -> (norm of the sum, the sum): the sum is the residual stream that goes on, x itself without a residual."""

    def __init__(self, features: int, eps: float = 1e-6, device=None, dtype=None):
        super().__init__()
        self.eps = float(eps)
        self.weight = torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype))

    def forward(self, x, residual=None):
        if residual is None:
            return _RMSNorm.apply(x, None, self.weight, self.eps), x
        x, residual = _beside_the_stream(x, residual)
        return _RMSNorm.apply(x, residual, self.weight, self.eps)


class DivisionNormLinear(torch.nn.Module):
    """forward(x, residual=None) -> (linear(norm of the sum), the sum), the linear layer's input cached in 8 bits."""

    def __init__(self, features: int, out_features: int, bias: bool = False, eps: float = 1e-6, code: str = "int8", group: int = 0, device=None,
                 dtype=None):
        super().__init__()
        if code not in ("int8", "e4m3"):
            raise ValueError("code is 'int8' or 'e4m3'")
        self.norm = DivisionRMSNorm(features, eps, device, dtype)
        self.linear = torch.nn.Linear(features, out_features, bias=bias, device=device, dtype=dtype)
        self.code, self.group = code, int(group)

    def forward(self, x, residual=None):
        args = (self.norm.weight, self.linear.weight, self.linear.bias, self.norm.eps, self.code, self.group)
        if residual is None:
            return _NormLinear.apply(x, None, *args), x
        x, residual = _beside_the_stream(x, residual)
        return _NormLinear.apply(x, residual, *args)


class _TokenLogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, top, ignore_index, overwrite):
        low = torch.empty(ids.shape, dtype=torch.float32, device=ids.device)
        f = division_log_probs(logits, ids, top=top, ignore_index=ignore_index, lse_low=low)
        ctx.save_for_backward(logits, ids, f.lse.view(-1), f.entropy.view(-1), low.view(-1))
        ctx.ignore_index, ctx.overwrite, ctx.overwritten = ignore_index, overwrite, False
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*(t for t in (f.lse, f.top_logp, f.top_ids) if t is not None))
        return tuple(f)

    @staticmethod
    @_first_derivatives
    def backward(ctx, grad_logp, grad_entropy, *rest):
        logits, ids, *per_row = ctx.saved_tensors
        lse, entropy, low = (t.view(ids.shape) for t in per_row)
        if grad_logp is None and grad_entropy is None:
            return None, None, None, None, None
        g = torch.zeros_like(lse) if grad_logp is None else grad_logp.contiguous()
        out = None
        if ctx.overwrite:
            if ctx.overwritten:                                 # torch itself does not look at the versions of what a saved-tensor hook has kept
                raise RuntimeError("the logits have been overwritten by an earlier backward pass")
            ctx.overwritten = True
            out = logits.detach()                               # shares their version: who saved them too is told that they are gone
        got = division_log_probs_backward(logits, ids, lse, g, entropy=entropy, grad_entropy=None if grad_entropy is None else grad_entropy.contiguous(),
                                          ignore_index=ctx.ignore_index, out=out, lse_low=low)
        return got, None, None, None, None


def division_token_log_probs(logits: torch.Tensor, ids: torch.Tensor, top: int = 0, ignore_index: int = -100, overwrite: bool = False) -> LogProbs:
    """division_log_probs with gradients through logp and the entropy.

    overwrite: the backward pass writes the gradient over the logits, which nothing else may need by then.  A second backward pass raises; so does that of an
    operation that saved the logits too, except under a saved-tensor hook, where torch does not see that they are gone."""
    lead = logits.shape[:-1]
    if logits.is_contiguous() and logits.dim() > 2 and logits.numel() > 0 and ids.shape == lead and ids.is_contiguous():
        # as rows: the saved-tensor hook keeps tensors of two dimensions as they are, and a softmax of rebuilt logits would be another one
        logits, ids = logits.view(-1, logits.shape[-1]), ids.view(-1)
    got = _TokenLogProbs.apply(logits, ids, int(top), int(ignore_index), bool(overwrite))
    return LogProbs._make(t if t is None else t.view((*lead, *t.shape[logits.dim() - 1:])) for t in got)
