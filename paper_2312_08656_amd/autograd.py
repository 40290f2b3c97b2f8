"""Autograd glue for one MaxK aggregation: Y = A * MaxK_k(H)  (training dataflow of Sec. 3.2, Eq. 2), and for a whole layer around it.

Forward : maxk_topk_cbsr -> maxk_spgemm_fwd.
Backward: maxk_sspmm_bwd (gradient only at the CBSR support) -> maxk_cbsr_scatter back to dense.
Every step runs in the HIP kernels; torch provides tensors, the stream and the autograd tape.  What the kernels write is not on the tape, so a second
derivative through either function is refused.

A layer, Y = A * MaxK_k(X W^T + b), keeps its input in 8 or 4 bits for the weight gradient, which is taken from the CBSR gradient and the
stored codes: neither X in 32 bits nor a dense dH is kept or made for it.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as _b
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
        if bits == 8:
            weights = (W,)
            H = torch.mm(X, W.t()) if b is None else torch.addmm(b, X, W.t())
        else:
            weights = _mx.mx_empty(dout, din, 4, X.device)
            _mx.maxk_mx_quantize(W, *weights)
            H = torch.empty((N, dout), dtype=torch.float32, device=X.device)
            _mx.maxk_mx_linear(*stored, *weights, H, None if b is None else b.contiguous())
        ib = 1 if dout <= 256 else 2 if dout <= 65536 else 4
        Y, sp_index = _b.aggregate_forward(graph, H, k, ib)
        ctx.graph, ctx.k, ctx.sizes, ctx.with_bias = graph, k, (N, din, dout), b is not None
        ctx.save_for_backward(sp_index, *stored, *weights)
        return Y

    @staticmethod
    @once_differentiable
    def backward(ctx, dY: torch.Tensor):
        sp_index, codes, scales, *weights = ctx.saved_tensors
        N, din, dout = ctx.sizes
        need_X, need_W, need_b = ctx.needs_input_grad[:3]
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
        return dX, dW if need_W else None, db, None, None, None, None


def maxk_layer(X: torch.Tensor, W: torch.Tensor, b: Optional[torch.Tensor], graph: _b.MaxKGraph, k: int, bits: int = 8) -> torch.Tensor:
    """Y = A * MaxK_k(X W^T + b) for X [N, din], W [dout, din], b [dout] or None (float32), differentiable (once) with respect to all three.

    Under autocast 16-bit arguments are widened, and the layer stays one of float32.

    bits=8: the product is torch's, in float32; X is kept in 8 bits, and dW is that of the kept values.
    bits=4: X and W are rounded to 4 bits, the product and both its gradients are of the rounded values (straight through the rounding).
    """
    return MaxKLayer.apply(X, W, b, graph, k, bits, torch.is_grad_enabled())  # (False within forward in any case)
