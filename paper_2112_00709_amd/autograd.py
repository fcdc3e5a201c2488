"""LF-MMI objective and a network's last layers as differentiable PyTorch functions on the GPU.

The network's output (pseudo-log-likelihoods, Sec. 3 of the paper) goes in, the
objective of Eq. 16 comes out; its derivative with respect to every network
output (Eq. 17: numerator minus denominator pdf posteriors) was already
computed by ``lfmmi_loss_grad`` in the forward call and is only scaled by the
incoming gradient in the backward call.  Splitting a batch into sub-batches and
calling ``backward`` once per sub-batch accumulates the parameter gradients of
the whole batch (the B/F scheme of the paper's training recipe), since the
objective is a sum over utterances.

``layer_norm``, ``residual_norm``, ``affine``, ``gated_affine``, ``token_logprobs``
and ``affine_logprobs`` are the operators of ``paper_2112_00709_amd.layers`` with
their gradients: what makes the network's output from hidden frames and takes the
objective's derivative back into the weights, and the frame log probabilities that
recipes use beside it.
"""
from __future__ import annotations

from typing import Optional

from . import Graph, fb_lfmmi_workspace_bytes, lfmmi_loss_grad


def _torch():
    import torch
    return torch


def _make_function():
    torch = _torch()

    class _LFMMI(torch.autograd.Function):
        @staticmethod
        def forward(ctx, emis, lengths, den, num, ws, lengths_host):
            if emis.dtype != torch.float32 or not emis.is_cuda:
                raise TypeError("emis must be a float32 tensor on the GPU")
            loss, zn, zd, grad = lfmmi_loss_grad(den, num, emis.contiguous(), lengths, ws=ws, lengths_host=lengths_host)
            ctx.save_for_backward(grad)
            ctx.mark_non_differentiable(zn, zd)
            return loss, zn, zd

        @staticmethod
        def backward(ctx, g_loss, _g_zn, _g_zd):
            (grad,) = ctx.saved_tensors
            return grad * g_loss.to(grad.dtype), None, None, None, None, None

    return _LFMMI


_fn = None


def lfmmi_loss(emis, lengths, den: Graph, num: Graph, ws: Optional[object] = None, lengths_host=None):
    """-> (loss [1] float64 (sum over utterances of log Z_num - log Z_den), logz_num [B], logz_den [B]).

    ``emis``: float32 CUDA tensor [B, N, D] that may require grad; ``lengths``: int32 CUDA tensor [B];
    ``den``: shared denominator graph; ``num``: packed numerator graphs of the same B utterances;
    ``ws``: optional reusable workspace (uint8 CUDA tensor of ``fb_lfmmi_workspace_bytes`` bytes);
    ``lengths_host``: optional host copy of ``lengths`` (the launches of the call are then scheduled by them).
    """
    global _fn
    if _fn is None:
        _fn = _make_function()
    return _fn.apply(emis, lengths, den, num, ws, lengths_host)


def workspace(den: Graph, num: Graph, B: int, N: int, D: int, device="cuda"):
    torch = _torch()
    return torch.empty((fb_lfmmi_workspace_bytes(den, num, B, N, D),), dtype=torch.uint8, device=device)


# ----------------------------------------------------------------- a network's last layers

_layer_fns = None


def _layer_functions():
    global _layer_fns
    if _layer_fns is not None:
        return _layer_fns
    torch = _torch()
    from torch.autograd.function import once_differentiable

    from . import layers as fl

    # `recording`: whether gradients are recorded where the function is called (inside of forward they never are, and
    # needs_input_grad does not look at it).  What only a backward pass reads is formed if one can follow.
    class _LayerNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, eps, recording):
            if not (recording and any(ctx.needs_input_grad[:3])):
                return fl.fb_layer_norm(x, weight, bias, eps)
            y, mean, rstd = fl.fb_layer_norm(x, weight, bias, eps, want_stats=True)
            ctx.save_for_backward(x, weight, mean, rstd)
            ctx.bias_dtype = None if bias is None else bias.dtype
            return y

        @staticmethod
        @once_differentiable
        def backward(ctx, dy):
            x, weight, mean, rstd = ctx.saved_tensors
            dx, dw, db = fl.fb_layer_norm_grad(dy.contiguous(), x, mean, rstd, weight, ctx.needs_input_grad[0], ctx.needs_input_grad[1],
                                               ctx.needs_input_grad[2])
            return dx, None if dw is None else dw.to(weight.dtype), None if db is None else db.to(ctx.bias_dtype), None, None

    class _Affine(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, residual, activation, out_dtype, recording):
            keep = recording and activation != "none" and any(ctx.needs_input_grad[:3])
            out = fl.fb_affine(x, weight, bias, activation, residual, out_dtype, want_preact=keep)
            y, preact = out if keep else (out, None)
            ctx.save_for_backward(x, weight, preact)
            ctx.activation = activation
            return y

        @staticmethod
        @once_differentiable
        def backward(ctx, dy):
            x, weight, preact = ctx.saved_tensors
            dy = dy.contiguous()
            dx = dw = db = None
            if any(ctx.needs_input_grad[:3]):
                dx, dw, db = fl.fb_affine_grad(dy, x, weight, ctx.activation, preact, *ctx.needs_input_grad[:3])
            return dx, dw, db, dy if ctx.needs_input_grad[3] else None, None, None, None

    class _TokenLogprobs(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, tokens, top, recording):
            logprobs, entropy, logz, ids, best = fl.fb_token_logprobs(logits, tokens, top)
            if recording and ctx.needs_input_grad[0]:      # (copies: the caller may change its results in place)
                ctx.save_for_backward(logits, tokens, logz.clone(), entropy.clone())
            ctx.mark_non_differentiable(logz, ids, best)
            ctx.set_materialize_grads(False)
            return logprobs, entropy, logz, ids, best

        @staticmethod
        @once_differentiable
        def backward(ctx, g_logprobs, g_entropy, _g_logz, _g_ids, _g_best):
            if g_logprobs is None and g_entropy is None:
                return None, None, None, None
            logits, tokens, logz, entropy = ctx.saved_tensors
            g = [None if t is None else t.contiguous() for t in (g_logprobs, g_entropy)]
            return fl.fb_token_logprobs_grad(logits, tokens, logz, entropy, *g), None, None, None

    class _ResidualNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h, residual, gate, inner_weight, inner_bias, weight, bias, scale, inner, outer, eps, recording):
            vectors = dict(scale=scale, inner=inner, inner_weight=inner_weight, inner_bias=inner_bias, outer=outer, weight=weight)
            ctx.set_materialize_grads(False)
            if not (recording and any(ctx.needs_input_grad[:7])):
                return fl.fb_residual_norm(h, residual, gate, bias=bias, eps=eps, **vectors)
            s, y, stats = fl.fb_residual_norm(h, residual, gate, bias=bias, eps=eps, want_stats=True, **vectors)
            # (s is what the backward pass reads of its outputs; without an outer norm it reads neither)
            ctx.save_for_backward(h, s if outer != "none" else None, stats, gate, inner_weight, inner_bias, weight)
            ctx.rest = scale, inner, outer, [None if t is None else t.dtype for t in (inner_weight, inner_bias, weight, bias)]
            return s, y

        @staticmethod
        @once_differentiable
        def backward(ctx, ds, dy):
            if ds is None and dy is None:
                return (None,) * 12
            h, s, stats, gate, inner_weight, inner_bias, weight = ctx.saved_tensors
            scale, inner, outer, dtypes = ctx.rest
            need = ctx.needs_input_grad
            ds, dy = [None if t is None else t.contiguous() for t in (ds, dy)]
            if dy is None and outer != "none":
                dy = torch.zeros_like(ds)
            dh, dr, dgate, *sums = fl.fb_residual_norm_grad(ds, dy, h, s, stats, gate, scale=scale, inner=inner, inner_weight=inner_weight,
                                                            inner_bias=inner_bias, outer=outer, weight=weight, want_dh=need[0], want_dresidual=need[1],
                                                            want_dgate=need[2], want_dinner=need[3] or need[4], want_douter=need[5] or need[6])
            sums = [g.to(dtype) if want else None for g, dtype, want in zip(sums, dtypes, need[3:7])]
            return dh, dr, None if dgate is None else dgate.to(gate.dtype), *sums, None, None, None, None, None

    class _GatedAffine(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, activation, recording):
            if not (recording and any(ctx.needs_input_grad[:3])):
                return fl.fb_gated_affine(x, weight, bias, activation)
            y, preact = fl.fb_gated_affine(x, weight, bias, activation, want_preact=True)
            ctx.save_for_backward(x, weight, preact)
            ctx.activation = activation
            return y

        @staticmethod
        @once_differentiable
        def backward(ctx, dy):
            x, weight, preact = ctx.saved_tensors
            return *fl.fb_gated_affine_grad(dy.contiguous(), x, weight, preact, ctx.activation, *ctx.needs_input_grad[:3]), None, None

    class _AffineLogprobs(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, tokens, recording):
            logprobs, entropy, logz = fl.fb_affine_logprobs(x, weight, tokens, bias)
            if recording and any(ctx.needs_input_grad[:3]):
                ctx.save_for_backward(x, weight, bias, tokens, logz.clone(), entropy.clone())
            ctx.mark_non_differentiable(logz)
            ctx.set_materialize_grads(False)
            return logprobs, entropy, logz

        @staticmethod
        @once_differentiable
        def backward(ctx, g_logprobs, g_entropy, _g_logz):
            if g_logprobs is None and g_entropy is None:
                return None, None, None, None, None
            x, weight, bias, tokens, logz, entropy = ctx.saved_tensors
            g = [None if t is None else t.contiguous() for t in (g_logprobs, g_entropy)]
            return *fl.fb_affine_logprobs_grad(x, weight, tokens, logz, entropy, *g, bias, *ctx.needs_input_grad[:3]), None, None

    _layer_fns = _LayerNorm, _Affine, _TokenLogprobs, _ResidualNorm, _GatedAffine, _AffineLogprobs
    return _layer_fns


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """``layers.fb_layer_norm`` with its gradient with respect to x, weight and bias."""
    return _layer_functions()[0].apply(x, weight, bias, eps, _torch().is_grad_enabled())


def affine(x, weight, bias=None, activation: str = "none", residual=None, out_dtype=None):
    """``layers.fb_affine`` with its gradient with respect to x, weight, bias and residual.  Where a gradient can
    follow, the forward call of an activation keeps what that was applied to, rounded to x's type."""
    return _layer_functions()[1].apply(x, weight, bias, residual, activation, out_dtype, _torch().is_grad_enabled())


def token_logprobs(logits, tokens, top: int = 0):
    """``layers.fb_token_logprobs`` -> (logprobs, entropy, logz, top_ids, top_logprobs); the first two have gradients with
    respect to the logits, the others do not."""
    return _layer_functions()[2].apply(logits, tokens, top, _torch().is_grad_enabled())


def residual_norm(h, residual=None, gate=None, scale: float = 1.0, inner: str = "none", inner_weight=None, inner_bias=None, outer: str = "layer",
                  weight=None, bias=None, eps: float = 1e-5):
    """``layers.fb_residual_norm`` -> (s, y), y None with outer "none", with its gradient with respect to h, residual, gate and the
    norms' weights and biases.  s is read again by the backward pass where there is an outer norm: it must not be changed in place then."""
    return _layer_functions()[3].apply(h, residual, gate, inner_weight, inner_bias, weight, bias, scale, inner, outer, eps, _torch().is_grad_enabled())


def gated_affine(x, weight, bias=None, activation: str = "silu"):
    """``layers.fb_gated_affine`` with its gradient with respect to x, weight and bias.  Where a gradient can follow, the forward
    call keeps both factors before the activation, rounded to x's type."""
    return _layer_functions()[4].apply(x, weight, bias, activation, _torch().is_grad_enabled())


def affine_logprobs(x, weight, tokens, bias=None):
    """``layers.fb_affine_logprobs`` -> (logprobs, entropy, logz); the first two have gradients with respect to x, weight and bias."""
    return _layer_functions()[5].apply(x, weight, bias, tokens, _torch().is_grad_enabled())
