"""The norm and distillation under autograd, the library's calls replaced by plain torch on the host: operands that autocast mixes, and a teacher that wants a gradient."""
import pytest
import torch

import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import autograd

HALVES = [torch.bfloat16, torch.float16]


def rms_norm(X, gamma, Y=None, codes=None, scales=None, residual=None, H=None, rstd=None, eps=1e-6):
    assert gamma.dtype == torch.float32 and Y.dtype == X.dtype and (residual is None or residual.dtype == X.dtype == H.dtype)
    h = X if residual is None else X + residual
    r = torch.rsqrt(h.float().square().mean(1) + eps)
    Y.copy_(h.float() * r[:, None] * gamma)
    rstd.copy_(r)
    if H is not None:
        H.copy_(h)


def rms_norm_grad(dY, H, gamma, rstd, dX, dgamma=None, dH=None, workspace=None):
    assert dY.dtype == H.dtype == dX.dtype and (dH is None or dH.dtype == H.dtype)
    x, g = H.float() * rstd[:, None], dY.float() * gamma
    dX.copy_(rstd[:, None] * (g - x * (g * x).mean(1, keepdim=True)) + (0.0 if dH is None else dH.float()))
    if dgamma is not None:
        dgamma.copy_((dY.float() * x).sum(0))


@pytest.fixture
def calls(monkeypatch):
    for name, plain in (("maxk_rms_norm", rms_norm), ("maxk_rms_norm_grad", rms_norm_grad), ("maxk_distill", lambda logits, data, index, loss, t: loss.zero_())):
        # a kernel's writes are not on the tape, and autocast does not change what it computes
        monkeypatch.setattr(autograd._heads, name, torch.no_grad()(torch.autocast("cpu", enabled=False)(plain)))


def operands(types):
    gen = torch.Generator().manual_seed(1)
    return [torch.randn(*s, generator=gen).to(t) for s, t in zip(((6, 16), (6, 16), (16,)), types)]


@pytest.mark.parametrize("half", HALVES, ids=str)
@pytest.mark.parametrize("mix", ["X", "residual", "gamma", "both"])
def test_operands_that_autocast_mixes(calls, mix, half):
    """They are taken in float32, as maxk_norm_layer and maxk_layer do; gradients have their operands' types."""
    f32 = torch.float32
    types = {"X": (half, f32, f32), "residual": (f32, half, f32), "gamma": (f32, f32, half), "both": (torch.bfloat16, torch.float16, f32)}[mix]
    X, R, gamma = operands(types)
    wide = [t.float().requires_grad_(True) for t in (X, R, gamma)]
    Y, H = maxk.maxk_residual_norm(wide[0], wide[2], wide[1])
    a, b = operands((f32, f32, f32))[:2]
    want = torch.autograd.grad([Y, H], wide, [a, b])
    given = [t.requires_grad_(True) for t in (X, R, gamma)]
    with torch.autocast("cpu", dtype=torch.bfloat16):
        Y2, H2 = maxk.maxk_residual_norm(given[0], given[2], given[1])
    assert torch.equal(Y2, Y) and torch.equal(H2, H) and Y2.dtype == f32
    got = torch.autograd.grad([Y2, H2], given, [a, b])
    assert [g.dtype for g in got] == [t.dtype for t in given]
    assert all(torch.equal(g, w.to(g.dtype)) for g, w in zip(got, want))
    with pytest.raises(maxk.MaxKError):
        maxk.maxk_residual_norm(given[0], given[2], given[1])  # as before, where autocast is off


@pytest.mark.parametrize("half", HALVES, ids=str)
def test_operands_of_one_type_stay_in_it_under_autocast(calls, half):
    X, R, gamma = operands((half, half, torch.float32))
    with torch.autocast("cpu", dtype=torch.bfloat16):
        Y, H = maxk.maxk_residual_norm(X, gamma, R)
        alone = maxk.maxk_residual_norm(X, gamma)
    assert Y.dtype == H.dtype == alone.dtype == half


@pytest.mark.gpu
@pytest.mark.parametrize("half", HALVES, ids=str)
def test_a_linear_map_and_a_residual_under_autocast_on_the_device(half):
    gen = torch.Generator(device="cuda").manual_seed(2)
    X, R, W = (torch.randn(s, generator=gen, device="cuda") for s in ((50, 40), (50, 72), (72, 40)))
    W.requires_grad_(True), R.requires_grad_(True)
    gamma = torch.ones(72, device="cuda", requires_grad=True)
    with torch.autocast("cuda", dtype=half):
        h = torch.nn.functional.linear(X, W)
        assert h.dtype == half
        Y, H = maxk.maxk_residual_norm(h, gamma, R)
    wide = [h.detach().float().requires_grad_(True), gamma, R]
    Y2, H2 = maxk.maxk_residual_norm(*wide)
    assert torch.equal(Y, Y2) and torch.equal(H, H2)
    got, want = torch.autograd.grad(Y.square().sum() + H.sum(), [h, gamma, R]), torch.autograd.grad(Y2.square().sum() + H2.sum(), wide)
    assert all(torch.equal(g, w.to(g.dtype)) for g, w in zip(got, want))


def test_a_teacher_that_wants_a_gradient_is_refused(calls):
    """The loss has none for it: what would be left out is said."""
    logits, top = torch.zeros(3, 5, requires_grad=True), torch.zeros(3, 2, requires_grad=True)
    index = torch.zeros(3, 2, dtype=torch.int32)
    with pytest.raises(maxk.MaxKError, match="detach"):
        maxk.maxk_distill_loss(logits, top, index)
    assert maxk.maxk_distill_loss(logits, top.detach(), index).requires_grad
    with torch.no_grad():
        maxk.maxk_distill_loss(logits, top, index)
    assert not maxk.maxk_distill_loss(logits.detach(), top.detach(), index).requires_grad
