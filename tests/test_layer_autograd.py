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
            # a kernel's writes are not on the tape, and autocast does not change what it computes
            monkeypatch.setattr(module, name, torch.no_grad()(torch.autocast("cpu", enabled=False)(getattr(stand_ins, name))))
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


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("given", [torch.float32, torch.bfloat16])
def test_the_layer_is_one_of_float32_under_autocast(calls, bits, given):
    X, W, b = _operands()
    x = X.detach().to(given)  # as a layer before it leaves it there
    dY = torch.randn(12, 24, generator=torch.Generator().manual_seed(3))
    plain = [x.float().requires_grad_(True), W, b]
    Y = maxk.maxk_layer(*plain, None, 8, bits)
    want = torch.autograd.grad(Y, plain, dY)
    args = [x.requires_grad_(True), W, b]
    with torch.autocast("cpu", dtype=torch.bfloat16):
        Y2 = maxk.maxk_layer(*args, None, 8, bits)
        inside = torch.autograd.grad(Y2, args, dY, retain_graph=True)
    outside = torch.autograd.grad(Y2, args, dY)
    assert torch.equal(Y2, Y)
    for got in (inside, outside):
        assert [g.dtype for g in got] == [given, torch.float32, torch.float32]
        assert all(torch.equal(g, w.to(g.dtype)) for g, w in zip(got, want))
    with pytest.raises(maxk.MaxKError):
        maxk.maxk_layer(X.detach().bfloat16(), W, b, None, 8, bits)  # as before, where autocast is off


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_the_layer_trains_under_autocast_on_the_device(bits):
    gen = torch.Generator(device="cuda").manual_seed(4)
    N, din, dout, k = 200, 40, 48, 8
    col = torch.randint(N, (N * 5,), generator=gen, device="cuda").to(torch.int32)
    graph = maxk.maxk_graph_create(torch.arange(0, 5 * N + 1, 5, device="cuda", dtype=torch.int32), col, torch.rand(N * 5, generator=gen, device="cuda"))
    X, W0, W, b = (torch.randn(s, generator=gen, device="cuda") for s in ((N, 30), (din, 30), (dout, din), (dout,)))
    W.requires_grad_(True), b.requires_grad_(True), W0.requires_grad_(True)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        h = torch.nn.functional.linear(X, W0)
        assert h.dtype == torch.bfloat16
        Y = maxk.maxk_layer(h, W, b, graph, k, bits)
    assert torch.equal(Y, maxk.maxk_layer(h.float(), W, b, graph, k, bits))
    want = torch.autograd.grad(maxk.maxk_layer(h.float(), W, b, graph, k, bits).square().sum(), [W, b])
    Y.square().sum().backward()
    assert torch.equal(W.grad, want[0]) and torch.equal(b.grad, want[1]) and bool(W0.grad.any())


@pytest.mark.parametrize("bits", [8, 4])
def test_a_bias_is_one_of_the_columns(calls, bits):
    X, W, b = (t.detach() for t in _operands())
    for bad in (b[:1], b[:-1], b[0], b.reshape(1, -1), b.expand(12, 24), b.double(), b.bfloat16()):
        with pytest.raises(maxk.MaxKError, match="maxk_layer: b must be"):
            maxk.maxk_layer(X, W, bad, None, 8, bits)
    strided = torch.stack([b, b], dim=1)[:, 0]
    assert torch.equal(maxk.maxk_layer(X, W, strided, None, 8, bits), maxk.maxk_layer(X, W, b, None, 8, bits))
    assert torch.isfinite(maxk.maxk_layer(X, W, None, None, 8, bits)).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_no_checkpoint_where_nothing_will_read_it(calls, bits):
    def made(needs, grad=True):
        calls.made.clear()
        with torch.set_grad_enabled(grad):
            Y = maxk.maxk_layer(*_operands(needs), None, 8, bits)
        quantized = calls.made.count("quantize")
        if Y.requires_grad:
            Y.sum().backward()
        return quantized, Y.detach()

    without = 0 if bits == 8 else 2  # in 4 bits the product itself reads the codes of X and W
    kept, Y = made((True, True, True))
    assert kept == without + (bits == 8)
    for needs, grad, count in (((False, False, False), True, without), ((True, False, False), True, without), ((True, True, True), False, without),
                               ((False, True, False), True, kept), ((False, False, True), True, kept)):
        got = made(needs, grad)
        assert got[0] == count, (needs, grad)
        assert torch.equal(got[1], Y)
