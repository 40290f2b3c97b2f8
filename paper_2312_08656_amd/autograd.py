"""Autograd glue for one MaxK aggregation: Y = A * MaxK_k(H)  (training dataflow of Sec. 3.2, Eq. 2), and for a whole layer around it.

Forward : maxk_topk_cbsr -> maxk_spgemm_fwd.
Backward: maxk_sspmm_bwd (gradient only at the CBSR support) -> maxk_cbsr_scatter back to dense.
Every step runs in the HIP kernels; torch provides tensors, the stream and the autograd tape.  What the kernels write is not on the tape, so a second
derivative through either function is refused.

A layer, Y = A * MaxK_k(X W^T + b), keeps its input in 8 or 4 bits for the weight gradient, which is taken from the CBSR gradient and the
stored codes: neither X in 32 bits nor a dense dH is kept or made for it.  With the norm in front of it (maxk_norm_layer) that input is written by the norm.

Behind the last layer: log probabilities and entropies of classes, and distillation from a teacher's largest logits, whose backward pass reads the logits again
and keeps nothing beside them.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as _b
from . import heads as _heads
from . import mx as _mx


class MaxKAggregate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, H: torch.Tensor, graph: _b.MaxKGraph, k: int, index_bytes: int = 0):
        N, dim = H.shape
        ib = index_bytes or (1 if dim <= 256 else 2 if dim <= 65536 else 4)
        Y, sp_index = _b.aggregate_forward(graph, H.contiguous(), k, ib)
        ctx.graph, ctx.dim, ctx.k = graph, dim, k
        ctx.save_for_backward(sp_index)
        return Y

    @staticmethod
    @once_differentiable
    def backward(ctx, dY: torch.Tensor):
        (sp_index,) = ctx.saved_tensors
        dH = _b.aggregate_backward(ctx.graph, dY.contiguous(), sp_index, ctx.dim, ctx.k)
        return dH, None, None, None


def maxk_aggregate(H: torch.Tensor, graph: _b.MaxKGraph, k: int) -> torch.Tensor:
    """Y = A * MaxK_k(H), differentiable (once) with respect to H."""
    return MaxKAggregate.apply(H, graph, k)


_HALVES = (torch.bfloat16, torch.float16)


class MaxKLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X: torch.Tensor, W: torch.Tensor, b: Optional[torch.Tensor], graph: _b.MaxKGraph, k: int, bits: int, tape: bool = True):
        if torch.is_autocast_enabled(X.device.type):
            with torch.autocast(X.device.type, enabled=False):
                return MaxKLayer.forward(ctx, *(t.float() if t is not None and t.dtype in _HALVES else t for t in (X, W, b)), graph, k, bits, tape)
        if X.dim() != 2 or W.dim() != 2 or X.shape[1] != W.shape[1] or X.dtype != torch.float32 or W.dtype != torch.float32:
            raise _b.MaxKError("maxk_layer: X [N, din] and W [dout, din] must be float32 matrices of one width")
        if b is not None and (b.shape != W.shape[:1] or b.dtype != torch.float32):
            raise _b.MaxKError("maxk_layer: b must be float32 [dout]")
        if bits not in (8, 4):
            raise _b.MaxKError("maxk_layer: bits must be 8 or 4")
        X, W = X.contiguous(), W.contiguous()
        (N, din), dout = X.shape, W.shape[0]
        stored = (None, None)
        if bits == 4 or (tape and any(ctx.needs_input_grad[1:3])):  # in 8 bits only dW and db read the codes
            stored = _mx.mx_empty(N, din, bits, X.device)
            _mx.maxk_mx_quantize(X, *stored)
        Y, sp_index, weights = _layer_forward(X, stored, W, b, graph, k, bits)
        ctx.graph, ctx.k, ctx.sizes, ctx.with_bias = graph, k, (N, din, dout), b is not None
        ctx.save_for_backward(sp_index, *stored, *weights)
        return Y

    @staticmethod
    @once_differentiable
    def backward(ctx, dY: torch.Tensor):
        return (*_layer_backward(ctx, dY, ctx.saved_tensors, ctx.needs_input_grad[:3]), None, None, None, None)


def _layer_forward(X: Optional[torch.Tensor], stored, W: torch.Tensor, b: Optional[torch.Tensor], graph: _b.MaxKGraph, k: int, bits: int):
    """(A * MaxK_k(X W^T + b), columns kept, W as the backward pass takes it), X in 32 bits (8) or as stored (4)."""
    dout, din = W.shape
    if bits == 8:
        weights = (W,)
        H = torch.mm(X, W.t()) if b is None else torch.addmm(b, X, W.t())
    else:
        weights = _mx.mx_empty(dout, din, 4, W.device)
        _mx.maxk_mx_quantize(W, *weights)
        H = torch.empty((stored[0].shape[0], dout), dtype=torch.float32, device=W.device)
        _mx.maxk_mx_linear(*stored, *weights, H, None if b is None else b.contiguous())
    ib = 1 if dout <= 256 else 2 if dout <= 65536 else 4
    Y, sp_index = _b.aggregate_forward(graph, H, k, ib)
    return Y, sp_index, weights


def _layer_backward(ctx, dY: torch.Tensor, saved, needs):
    """(dX, dW, db) of those that are needed, from (columns kept, codes, scales, weights)."""
    sp_index, codes, scales, *weights = saved
    N, din, dout = ctx.sizes
    need_X, need_W, need_b = needs
    dX = dW = db = None
    dXs = torch.empty((N, ctx.k), dtype=torch.float32, device=dY.device)
    _b.maxk_sspmm_bwd(ctx.graph, dY.contiguous(), sp_index, dXs)
    if need_W or need_b:
        dW = torch.empty((dout, din), dtype=torch.float32, device=dY.device)
        db = torch.empty((dout,), dtype=torch.float32, device=dY.device) if ctx.with_bias and need_b else None
        _mx.maxk_mx_weight_grad_cbsr(codes, scales, dXs, sp_index, dW, db)
    if need_X:
        dX = torch.empty((N, din), dtype=torch.float32, device=dY.device)
        if len(weights) == 2:
            _mx.maxk_mx_input_grad_cbsr(dXs, sp_index, *weights, dX)
        else:
            dH = torch.empty((N, dout), dtype=torch.float32, device=dY.device)
            _b.maxk_cbsr_scatter(dXs, sp_index, dH)
            torch.mm(dH, weights[0], out=dX)
    return dX, dW if need_W else None, db


def maxk_layer(X: torch.Tensor, W: torch.Tensor, b: Optional[torch.Tensor], graph: _b.MaxKGraph, k: int, bits: int = 8) -> torch.Tensor:
    """Y = A * MaxK_k(X W^T + b) for X [N, din], W [dout, din], b [dout] or None (float32), differentiable (once) with respect to all three.

    Under autocast 16-bit arguments are widened, and the layer stays one of float32.

    bits=8: the product is torch's, in float32; X is kept in 8 bits, and dW is that of the kept values.
    bits=4: X and W are rounded to 4 bits, the product and both its gradients are of the rounded values (straight through the rounding).
    """
    return MaxKLayer.apply(X, W, b, graph, k, bits, torch.is_grad_enabled())  # (False within forward in any case)


def _norm_arguments(X, gamma, residual, what):
    if X.dim() != 2 or X.dtype not in _b._VALUE_TYPE or gamma.dtype != torch.float32 or gamma.shape != X.shape[1:]:
        raise _b.MaxKError(f"{what}: X must be a matrix [N, dim] of float32, bfloat16 or float16, gamma float32 [dim]")
    if residual is not None and (residual.shape != X.shape or residual.dtype != X.dtype):
        raise _b.MaxKError(f"{what}: the residual must be of X's shape and type")
    return X.contiguous(), gamma.contiguous(), None if residual is None else residual.contiguous()


def _norm_backward(dY, dH, H, gamma, rstd, needs):
    """(gradient of X and of the residual, dgamma) of those that are needed (of X, of gamma); dY or dH may be None."""
    need_X, need_gamma = needs
    if dY is None:  # only H is used
        return dH if need_X else None, torch.zeros_like(gamma) if need_gamma else None
    dX = torch.empty_like(H)
    dgamma = torch.empty_like(gamma) if need_gamma else None
    _heads.maxk_rms_norm_grad(dY.contiguous(), H, gamma, rstd, dX, dgamma, dH=None if dH is None else dH.contiguous())
    return dX if need_X else None, dgamma


class MaxKRMSNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X: torch.Tensor, gamma: torch.Tensor, residual: Optional[torch.Tensor], eps: float):
        if torch.is_autocast_enabled(X.device.type):
            gamma = gamma.float() if gamma.dtype in _HALVES else gamma
            if residual is not None and residual.dtype != X.dtype:
                X, residual = (t.float() if t.dtype in _HALVES else t for t in (X, residual))
        X, gamma, residual = _norm_arguments(X, gamma, residual, "maxk_residual_norm")
        Y, rstd = torch.empty_like(X), torch.empty(X.shape[0], dtype=torch.float32, device=X.device)
        H = None if residual is None else torch.empty_like(X)
        _heads.maxk_rms_norm(X, gamma, Y, residual=residual, H=H, rstd=rstd, eps=eps)
        ctx.save_for_backward(X if H is None else H, gamma, rstd)
        ctx.set_materialize_grads(False)
        return (Y,) if H is None else (Y, H)

    @staticmethod
    @once_differentiable
    def backward(ctx, dY: Optional[torch.Tensor], dH: Optional[torch.Tensor] = None):
        if dY is None and dH is None:
            return None, None, None, None
        need_X, need_gamma, need_residual = ctx.needs_input_grad[:3]
        dX, dgamma = _norm_backward(dY, dH, *ctx.saved_tensors, (need_X or need_residual, need_gamma))
        return dX if need_X else None, dgamma, dX if need_residual else None, None


def maxk_residual_norm(X: torch.Tensor, gamma: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6):
    """Y = H r gamma with H = X + residual and r = 1 / sqrt(mean of a row's H^2 + eps): (Y, H), or Y alone where there is no residual.  X and residual [N, dim] in
    float32, bfloat16 or float16, gamma float32 [dim]; differentiable (once) with respect to all three.  Under autocast an X and a residual of different types, and a
    gamma in 16 bits, are taken in float32."""
    out = MaxKRMSNorm.apply(X, gamma, residual, eps)
    return out[0] if residual is None else out


class MaxKNormLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X: torch.Tensor, residual: Optional[torch.Tensor], gamma: torch.Tensor, W: torch.Tensor, b: Optional[torch.Tensor], graph: _b.MaxKGraph,
                k: int, bits: int, eps: float, tape: bool = True):
        if torch.is_autocast_enabled(X.device.type):
            with torch.autocast(X.device.type, enabled=False):
                X, residual, gamma, W, b = (t.float() if t is not None and t.dtype in _HALVES else t for t in (X, residual, gamma, W, b))
                return MaxKNormLayer.forward(ctx, X, residual, gamma, W, b, graph, k, bits, eps, tape)
        if X.dtype != torch.float32 or W.dim() != 2 or W.dtype != torch.float32 or X.dim() != 2 or X.shape[1] != W.shape[1]:
            raise _b.MaxKError("maxk_norm_layer: X [N, din] and W [dout, din] must be float32 matrices of one width")
        if b is not None and (b.shape != W.shape[:1] or b.dtype != torch.float32):
            raise _b.MaxKError("maxk_norm_layer: b must be float32 [dout]")
        if bits not in (8, 4):
            raise _b.MaxKError("maxk_norm_layer: bits must be 8 or 4")
        X, gamma, residual = _norm_arguments(X, gamma, residual, "maxk_norm_layer")
        W = W.contiguous()
        N, din = X.shape
        stored = (None, None)
        if bits == 4 or (tape and any(ctx.needs_input_grad[3:5])):
            stored = _mx.mx_empty(N, din, bits, X.device)
        Y = torch.empty_like(X) if bits == 8 else None  # (4 bits: the codes carry the product)
        H = None if residual is None else torch.empty_like(X)
        rstd = torch.empty(N, dtype=torch.float32, device=X.device)
        _heads.maxk_rms_norm(X, gamma, Y, *stored, residual=residual, H=H, rstd=rstd, eps=eps)
        out, sp_index, weights = _layer_forward(Y, stored, W, b, graph, k, bits)
        ctx.graph, ctx.k, ctx.sizes, ctx.with_bias = graph, k, (N, din, W.shape[0]), b is not None
        ctx.save_for_backward(X if H is None else H, gamma, rstd, sp_index, *stored, *weights)
        ctx.set_materialize_grads(False)
        return (out,) if H is None else (out, H)

    @staticmethod
    @once_differentiable
    def backward(ctx, dOut: Optional[torch.Tensor], dH: Optional[torch.Tensor] = None):
        if dOut is None and dH is None:
            return (None,) * 10
        need_X, need_residual, need_gamma, need_W, need_b = ctx.needs_input_grad[:5]
        H, gamma, rstd, *saved = ctx.saved_tensors
        dY = dW = db = None
        if dOut is not None:
            dY, dW, db = _layer_backward(ctx, dOut, saved, (need_X or need_residual or need_gamma, need_W, need_b))
        elif need_W or need_b:  # only H is used
            dW = torch.zeros(ctx.sizes[2], ctx.sizes[1], device=H.device) if need_W else None
            db = torch.zeros(ctx.sizes[2], device=H.device) if need_b and ctx.with_bias else None
        dX = dgamma = None
        if need_X or need_residual or need_gamma:
            dX, dgamma = _norm_backward(dY, dH, H, gamma, rstd, (need_X or need_residual, need_gamma))
        return dX if need_X else None, dX if need_residual else None, dgamma, dW, db, None, None, None, None, None


def maxk_norm_layer(X: torch.Tensor, residual: Optional[torch.Tensor], gamma: torch.Tensor, W: torch.Tensor, b: Optional[torch.Tensor], graph: _b.MaxKGraph,
                    k: int, bits: int = 8, eps: float = 1e-6):
    """maxk_layer with the norm in front of it: (A * MaxK_k(Y W^T + b), H) with Y and H as of maxk_residual_norm, or the first alone where there is no residual.
    Everything is float32 and differentiable (once).  Y is written in 8 or 4 bits, as the layer keeps it, by the norm itself; bits as for maxk_layer."""
    out = MaxKNormLayer.apply(X, residual, gamma, W, b, graph, k, bits, eps, torch.is_grad_enabled())
    return out[0] if residual is None else out


class MaxKLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits: torch.Tensor, labels: Optional[torch.Tensor]):
        logits = logits.contiguous()
        labels = None if labels is None else labels.contiguous()
        logprob, entropy = (torch.empty(logits.shape[:1], dtype=torch.float32, device=logits.device) for _ in range(2))
        _heads.maxk_logprobs(logits, labels, None if labels is None else logprob, entropy)
        ctx.save_for_backward(logits, labels)
        ctx.set_materialize_grads(False)
        return (entropy,) if labels is None else (logprob, entropy)

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads: Optional[torch.Tensor]):
        logits, labels = ctx.saved_tensors
        dlogprob, dentropy = (g if g is None else g.contiguous() for g in ((None, *grads) if labels is None else grads))
        if dlogprob is None and dentropy is None:
            return None, None
        dlogits = torch.empty_like(logits)
        _heads.maxk_logprobs_grad(logits, dlogits, labels, dlogprob, dentropy)
        return dlogits, None


def maxk_class_logprobs(logits: torch.Tensor, labels: Optional[torch.Tensor]):
    """(log probability of each row's class in labels [N], entropy of each row), float32 [N], of logits [N, V] in float32, bfloat16 or float16; the
    entropies alone without labels.  A negative label is no class: 0, and no gradient.  Differentiable (once) with respect to the logits."""
    out = MaxKLogprobs.apply(logits, labels)
    return out[0] if labels is None else out


class MaxKDistill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits: torch.Tensor, top_data: torch.Tensor, top_index: torch.Tensor, temperature: float):
        logits, top_data, top_index = logits.contiguous(), top_data.contiguous(), top_index.contiguous()
        loss = torch.empty(logits.shape[:1], dtype=torch.float32, device=logits.device)
        _heads.maxk_distill(logits, top_data, top_index, loss, temperature)
        ctx.save_for_backward(logits, top_data, top_index)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss: torch.Tensor):
        logits, top_data, top_index = ctx.saved_tensors
        dlogits = torch.empty_like(logits)
        _heads.maxk_distill_grad(logits, top_data, top_index, dloss.contiguous(), dlogits, ctx.temperature)
        return dlogits, None, None, None


def maxk_distill_loss(logits: torch.Tensor, top_data: torch.Tensor, top_index: torch.Tensor, temperature: float = 1.0) -> torch.Tensor:
    """Divergence [N] (float32) of softmax(logits / temperature) from the softmax of a teacher's largest logits / temperature, as maxk_topk_cbsr or maxk_logprobs leaves
    them: top_data [N, k] at the columns top_index [N, k].  Differentiable (once) with respect to the logits; a top_data that requires a gradient is refused."""
    if torch.is_grad_enabled() and top_data.requires_grad:
        raise _b.MaxKError("maxk_distill_loss: there is no gradient of top_data: detach() it")
    return MaxKDistill.apply(logits, top_data, top_index, temperature)
