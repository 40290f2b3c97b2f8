"""A whole layer that keeps its input in 8 or 4 bits: forward, gradients, refusals, and the example that trains with it."""
import importlib.util
from pathlib import Path

import numpy as np
import pytest
import torch

import mx_common as mx
import paper_2312_08656_amd as maxk

pytestmark = pytest.mark.gpu


def _graph(N, gen):
    degree = torch.randint(0, 12, (N,), generator=gen, device="cuda")
    rowptr = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    rowptr[1:] = torch.cumsum(degree, 0)
    nnz = int(rowptr[-1])
    col = torch.randint(N, (nnz,), generator=gen, device="cuda").to(torch.int32)
    return maxk.maxk_graph_create(rowptr, col, torch.randn(nnz, generator=gen, device="cuda"))


def _stored(X, bits):
    return torch.from_numpy(mx.values(*mx.quantize(X.detach().cpu().numpy(), bits), X.shape[1])).cuda()


@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("N,din,dout,k", [(300, 100, 64, 8), (700, 256, 300, 32), (65, 33, 17, 17)])
def test_layer(N, din, dout, k, bits, with_bias):
    gen = torch.Generator(device="cuda").manual_seed(N + bits)
    graph = _graph(N, gen)
    X = torch.randn(N, din, generator=gen, device="cuda", requires_grad=True)
    W = (torch.randn(dout, din, generator=gen, device="cuda") / din ** 0.5).requires_grad_(True)
    b = torch.randn(dout, generator=gen, device="cuda", requires_grad=True) if with_bias else None
    dY = torch.randn(N, dout, generator=gen, device="cuda")
    Y = maxk.maxk_layer(X, W, b, graph, k, bits)
    dX, dW, *rest = torch.autograd.grad(Y, [X, W] + ([b] if with_bias else []), dY)

    # the steps one by one: H as the layer makes it, then the aggregation and its gradient at H
    H = torch.empty(N, dout, device="cuda")
    if bits == 8:
        H = torch.mm(X.detach(), W.detach().t()) if b is None else torch.addmm(b.detach(), X.detach(), W.detach().t())
        Wv = W.detach().double()
    else:
        xs, ws = maxk.mx_empty(N, din, 4), maxk.mx_empty(dout, din, 4)
        maxk.maxk_mx_quantize(X.detach(), *xs)
        maxk.maxk_mx_quantize(W.detach(), *ws)
        maxk.maxk_mx_linear(*xs, *ws, H, None if b is None else b.detach())
        Wv = _stored(W, 4)
    H.requires_grad_(True)
    Y2 = maxk.maxk_aggregate(H, graph, k)
    assert torch.equal(Y, Y2)
    (dH,) = torch.autograd.grad(Y2, H, dY)
    dH = dH.double().cpu()  # (sums of products in 64 bits on the host)
    Xv, Wv = _stored(X, bits).cpu(), Wv.cpu()
    for got, want, terms, n in ((dW, dH.t() @ Xv, dH.abs().t() @ Xv.abs(), N), (dX, dH @ Wv, dH.abs() @ Wv.abs(), dout)) + \
            (((rest[0], dH.sum(0), dH.abs().sum(0), N),) if with_bias else ()):
        bound = (8 + n ** 0.5) * 2.0 ** -24 * terms + 1e-30
        assert bool(((got.double().cpu() - want).abs() <= bound).all())


def test_only_what_is_asked_for():
    gen = torch.Generator(device="cuda").manual_seed(9)
    graph = _graph(200, gen)
    X, W, b = torch.randn(200, 40, generator=gen, device="cuda"), torch.randn(48, 40, generator=gen, device="cuda"), torch.randn(48, generator=gen, device="cuda")
    for bits in (8, 4):
        for needs in ((False, True, False), (True, False, False), (False, False, True)):
            args = [t.clone().requires_grad_(n) for t, n in zip((X, W, b), needs)]
            Y = maxk.maxk_layer(*args, graph, 8, bits)
            Y.backward(torch.ones_like(Y))
            assert [a.grad is not None for a in args] == list(needs)
    for bad in (lambda: maxk.maxk_layer(X, W, b, graph, 8, 16), lambda: maxk.maxk_layer(X[:, :-1], W, b, graph, 8), lambda: maxk.maxk_layer(X.half(), W, b, graph, 8)):
        with pytest.raises(maxk.MaxKError):
            bad()


def test_the_example_learns_and_keeps_less():
    path = Path(__file__).resolve().parent.parent / "examples" / "train_layers.py"
    spec = importlib.util.spec_from_file_location("train_layers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    kept = {}
    for bits in (32, 8, 4):
        losses, kept[bits] = example.train(bits, nodes=3000, degree=10, steps=25)
        assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0], (bits, losses[0], losses[-1])
    # inputs of 100 and 256 columns: 1424 bytes a node in 32 bits, 396 in 8, 204 in 4 (with scales and whole blocks), and k columns of a byte each
    assert kept[32] == 3000 * (1424 + 64) and kept[8] == 3000 * (128 + 4 + 256 + 8 + 64)
    assert kept[4] == 3000 * (64 + 4 + 128 + 8 + 64) + 256 * (64 + 4 + 128 + 8)
