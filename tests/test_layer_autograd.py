"""maxk_aggregate and maxk_layer under autograd, the library's calls replaced by plain torch on the host: what the functions hand back, not the kernels."""
import numpy as np
import pytest
import torch

import mx_common as mx
import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import autograd


class _Calls:
    """Plain forms of the calls that autograd.py makes, and the names of those that were made."""

    def __init__(self, N):
        self.A = torch.rand(N, N, generator=torch.Generator().manual_seed(1))
        self.made = []

    def aggregate_forward(self, graph, H, k, index_bytes):
        assert H.dtype == torch.float32
        self.made.append("forward")
        index = H.topk(k, dim=1).indices.sort(dim=1).values
        kept = torch.zeros_like(H).scatter(1, index, H.gather(1, index))
        return self.A @ kept, index.to(torch.int32)

    def maxk_sspmm_bwd(self, graph, dY, index, dXs):
        dXs.copy_((self.A.t() @ dY).gather(1, index.long()))

    def maxk_cbsr_scatter(self, values, index, dense):
        dense.zero_().scatter_(1, index.long(), values)

    def aggregate_backward(self, graph, dY, index, dim, k):
        dXs, dH = torch.empty(dY.shape[0], k), torch.empty(dY.shape[0], dim)
        self.maxk_sspmm_bwd(graph, dY, index, dXs)
        self.maxk_cbsr_scatter(dXs, index, dH)
        return dH

    def maxk_mx_quantize(self, X, codes, scales):
        assert X.dtype == torch.float32
        self.made.append("quantize")
        c, s = mx.quantize(X.detach().numpy(), 8 if codes.dtype == torch.int8 else 4)
        codes.copy_(torch.from_numpy(c)), scales.copy_(torch.from_numpy(s))

    @staticmethod
    def values(codes, scales, din):
        return torch.from_numpy(mx.values(codes.numpy(), scales.numpy(), din)).float()

    def maxk_mx_linear(self, xc, xs, wc, ws, Y, bias=None):
        din = 32 * xs.shape[1]
        Y.copy_(self.values(xc, xs, din) @ self.values(wc, ws, din).t() + (0.0 if bias is None else bias))

    def maxk_mx_weight_grad_cbsr(self, codes, scales, dXs, index, dW, db=None, workspace=None):
        self.made.append("weight_grad")
        dH = torch.from_numpy(mx.scatter(dXs.numpy(), index.numpy(), dW.shape[0])).float()
        dW.copy_(dH.t() @ self.values(codes, scales, dW.shape[1]))
        if db is not None:
            db.copy_(dH.sum(0))

    def maxk_mx_input_grad_cbsr(self, dXs, index, wc, ws, dX):
        dH = torch.from_numpy(mx.scatter(dXs.numpy(), index.numpy(), wc.shape[0])).float()
        dX.copy_(dH @ self.values(wc, ws, dX.shape[1]))


@pytest.fixture
def calls(monkeypatch):
    stand_ins = _Calls(12)
    for module, names in ((autograd._b, ("aggregate_forward", "aggregate_backward", "maxk_sspmm_bwd", "maxk_cbsr_scatter")),
                          (autograd._mx, ("maxk_mx_quantize", "maxk_mx_linear", "maxk_mx_weight_grad_cbsr", "maxk_mx_input_grad_cbsr"))):
        for name in names:
            monkeypatch.setattr(module, name, torch.no_grad()(getattr(stand_ins, name)))  # (a kernel's writes are not on the tape)
    return stand_ins


def _operands(needs=(True, True, True), N=12, din=40, dout=24):
    gen = torch.Generator().manual_seed(2)
    X, W, b = torch.randn(N, din, generator=gen), torch.randn(dout, din, generator=gen) / din ** 0.5, torch.randn(dout, generator=gen)
    return [t.requires_grad_(n) for t, n in zip((X, W, b), needs)]


def _penalised(Y, inputs):
    """A loss with a penalty on its gradients, whose own gradient needs second derivatives."""
    loss = (Y * Y).sum()
    return loss + sum((g * g).sum() for g in torch.autograd.grad(loss, inputs, create_graph=True))


def test_second_derivatives_of_the_aggregation_are_refused(calls):
    H = _operands()[0]
    first = torch.autograd.grad(maxk.maxk_aggregate(H, None, 8).sum(), H)[0]
    with pytest.raises(RuntimeError, match="once_differentiable"):
        _penalised(maxk.maxk_aggregate(H, None, 8), [H]).backward()
    assert torch.equal(torch.autograd.grad(maxk.maxk_aggregate(H, None, 8).sum(), H, create_graph=True)[0], first)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("needs", [(True, True, True), (True, False, False), (False, True, False), (False, True, True)])
def test_second_derivatives_of_the_layer_are_refused(calls, bits, needs):
    args = _operands(needs)
    wanted = [a for a in args if a.requires_grad]
    first = torch.autograd.grad(maxk.maxk_layer(*args, None, 8, bits).sum(), wanted)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        _penalised(maxk.maxk_layer(*args, None, 8, bits), wanted).backward()
    again = torch.autograd.grad(maxk.maxk_layer(*args, None, 8, bits).sum(), wanted, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
