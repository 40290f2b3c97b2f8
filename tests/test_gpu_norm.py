"""The residual norm and its gradients against 64 bits: every form of a row, every type, stored output bit for bit."""
import numpy as np
import pytest
import torch

import heads_common as hc
import paper_2312_08656_amd as maxk

pytestmark = pytest.mark.gpu
EPS = 1e-6


def inputs(N, dim, dtype, seed, residual=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    X = (randn(N, dim) * torch.exp(randn(N, 1))).to(dtype)
    R = randn(N, dim).to(dtype) if residual else None
    if N > 3:
        X[2] = 0
        if residual:
            R[2] = 0
    return X, R, 1 + 0.3 * randn(dim), randn


# one width for each number of lanes and units that a row may take, whole and ragged, and the widest
WIDTHS = [1, 7, 16, 33, 64, 100, 127, 200, 256, 300, 384, 500, 512, 700, 1000, 1024, 1433, 2048, 2500, 4096, 5003, 8192, 9001, 16384]


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("dim", WIDTHS)
def test_norm(dim, dtype):
    N = 67 if dim < 3000 else 5
    for residual in (True, False):
        X, R, gamma, _ = inputs(N, dim, dtype, dim, residual)
        H = torch.full_like(X, 7) if residual else None
        Y, rstd = torch.full_like(X, 7), torch.empty(N, device="cuda")
        maxk.maxk_rms_norm(X, gamma, Y, residual=R, H=H, rstd=rstd, eps=EPS)
        want_H, r, y = hc.norm(X, R, gamma, EPS)
        if residual:
            assert torch.equal(H, want_H)
        hc.close(rstd, r[:, 0], 2 * hc.U * r[:, 0])
        hc.close(Y, y, 4 * hc.U * np.abs(y), dtype)  # r, and two products


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim", [1, 31, 32, 64, 100, 130, 256, 384, 511, 768, 1000, 1500, 2048, 4100, 8192, 10000])
def test_stored_norm(dim, bits, dtype):
    N = 37 if dim < 3000 else 5
    X, R, gamma, _ = inputs(N, dim, dtype, dim + bits)
    codes, scales = maxk.mx_empty(N, dim, bits)
    codes.fill_(77), scales.fill_(77)
    H, Y = torch.empty_like(X), torch.empty_like(X)
    maxk.maxk_rms_norm(X, gamma, codes=codes, scales=scales, residual=R, H=H, eps=EPS)
    want_codes, want_scales = hc.stored(H, gamma, EPS, bits)
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)
    if dtype == torch.float32:  # the same as storing Y
        both, s = maxk.mx_empty(N, dim, bits)
        maxk.maxk_rms_norm(X, gamma, Y, both, s, R, H, eps=EPS)
        assert torch.equal(both, codes) and torch.equal(s, scales)
        maxk.maxk_mx_quantize(Y, both, s)
        assert torch.equal(both, codes) and torch.equal(s, scales)


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("dim", WIDTHS)
def test_norm_grad(dim, dtype):
    N = 131 if dim < 3000 else 5
    X, R, gamma, randn = inputs(N, dim, dtype, dim + 1)
    H, rstd = torch.empty_like(X), torch.empty(N, device="cuda")
    maxk.maxk_rms_norm(X, gamma, torch.empty_like(X), residual=R, H=H, rstd=rstd, eps=EPS)
    dY, dH = randn(N, dim).to(dtype), randn(N, dim).to(dtype)
    for arrives in (dH, None):
        dX, dgamma = torch.full_like(X, 7), torch.full((dim,), 7.0, device="cuda")
        maxk.maxk_rms_norm_grad(dY, H, gamma, rstd, dX, dgamma, dH=arrives)
        dx, bound, dg, size = hc.norm_grad(dY, H, gamma, rstd, arrives)
        hc.close(dX, dx, bound, dtype)
        hc.close(dgamma, dg, (N + 4) * hc.U * size)
        again = torch.empty_like(X)
        maxk.maxk_rms_norm_grad(dY, H, gamma, rstd, again, dH=arrives)
        assert torch.equal(again, dX)


@pytest.mark.parametrize("N,dim", [(1, 64), (9000, 48), (70000, 8), (2500, 300), (2100, 2100)])
def test_many_rows(N, dim):
    """Several rounds of a workgroup, partial sums of many of them; two calls give the same bits."""
    X, R, gamma, randn = inputs(N, dim, torch.float32, N)
    H, Y, rstd = torch.empty_like(X), torch.empty_like(X), torch.empty(N, device="cuda")
    maxk.maxk_rms_norm(X, gamma, Y, residual=R, H=H, rstd=rstd, eps=EPS)
    _, r, y = hc.norm(X, R, gamma, EPS)
    hc.close(Y, y, 4 * hc.U * np.abs(y))
    dY = randn(N, dim)
    outs = []
    for _ in range(2):
        dX, dgamma = torch.empty_like(X), torch.empty(dim, device="cuda")
        maxk.maxk_rms_norm_grad(dY, H, gamma, rstd, dX, dgamma)
        outs.append((dX, dgamma))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    dx, bound, dg, size = hc.norm_grad(dY, H, gamma, rstd, None)
    hc.close(dX, dx, bound)
    # a lane adds up its rows, at most ceil(N / 1024) of them, and up to 64 teams' sums; workgroups are added in 64 bits
    hc.close(dgamma, dg, (-(-N // 1024) + 64 + 4) * hc.U * size)


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
def test_in_place_and_offsets(dtype):
    """Results in the operands' own memory; operands that start at any element; nothing is written around them."""
    N, dim = 35, 77
    X, R, gamma, randn = inputs(N, dim, dtype, 5)
    H, Y, rstd = torch.empty_like(X), torch.empty_like(X), torch.empty(N, device="cuda")
    maxk.maxk_rms_norm(X, gamma, Y, residual=R, H=H, rstd=rstd, eps=EPS)
    for at in range(1, 4):
        flat = torch.full((N * dim + 8,), 3.0, dtype=dtype, device="cuda")
        mine = flat[at:at + N * dim].view(N, dim)
        mine.copy_(R)
        out = torch.full((N * dim + 8,), 3.0, dtype=dtype, device="cuda")
        y = out[at + 1:at + 1 + N * dim].view(N, dim)
        maxk.maxk_rms_norm(X, gamma, y, residual=mine, H=mine, eps=EPS)
        assert torch.equal(mine, H) and torch.equal(y, Y)
        assert (flat[:at] == 3).all() and (flat[at + N * dim:] == 3).all()
        assert (out[:at + 1] == 3).all() and (out[at + 1 + N * dim:] == 3).all()
    x = X.clone()
    maxk.maxk_rms_norm(x, gamma, Y, residual=R, H=x, eps=EPS)
    assert torch.equal(x, H)
    dY, dH, dX = randn(N, dim).to(dtype), randn(N, dim).to(dtype), torch.empty_like(X)
    maxk.maxk_rms_norm_grad(dY, H, gamma, rstd, dX, dH=dH)
    a, b = dY.clone(), dH.clone()
    maxk.maxk_rms_norm_grad(a, H, gamma, rstd, a, dH=dH)
    maxk.maxk_rms_norm_grad(dY, H, gamma, rstd, b, dH=b)
    assert torch.equal(a, dX) and torch.equal(b, dX)


def test_gradients_are_differences():
    """dX and dgamma against central differences of the 64-bit definition."""
    N, dim = 6, 20
    X, R, gamma, randn = inputs(N, dim, torch.float32, 11)
    X[2] = randn(dim)
    H, rstd = torch.empty_like(X), torch.empty(N, device="cuda")
    maxk.maxk_rms_norm(X, gamma, torch.empty_like(X), residual=R, H=H, rstd=rstd, eps=EPS)
    dY, dH = randn(N, dim), randn(N, dim)
    dX, dgamma = torch.empty_like(X), torch.empty(dim, device="cuda")
    maxk.maxk_rms_norm_grad(dY, H, gamma, rstd, dX, dgamma, dH=dH)

    def value(h, gam):
        r = 1 / np.sqrt((h * h).mean(axis=1, keepdims=True) + EPS)
        return (h * r * gam * hc.f64(dY)).sum() + (h * hc.f64(dH)).sum()

    h, gam, step = hc.f64(H), hc.f64(gamma), 1e-5
    for n, i in ((0, 0), (2, 7), (5, 19), (3, 4)):
        up, down = h.copy(), h.copy()
        up[n, i] += step
        down[n, i] -= step
        assert abs((value(up, gam) - value(down, gam)) / (2 * step) - dX[n, i].item()) < 1e-5  # the third derivative's step^2, and fp32
        up, down = gam.copy(), gam.copy()
        up[i] += step
        down[i] -= step
        assert abs((value(h, up) - value(h, down)) / (2 * step) - dgamma[i].item()) < 1e-5


def test_extremes_and_non_finite():
    dim = 40
    X = torch.ones(6, dim, device="cuda")
    X[0] = 0
    X[1] = 1e30
    X[2] = 1e-30
    X[3, 5] = float("nan")
    X[4, 6] = float("inf")
    gamma = torch.ones(dim, device="cuda")
    Y, rstd = torch.empty_like(X), torch.empty(6, device="cuda")
    codes, scales = maxk.mx_empty(6, dim, 8)
    maxk.maxk_rms_norm(X, gamma, Y, codes, scales, rstd=rstd, eps=EPS)
    assert (Y[0] == 0).all() and torch.allclose(Y[1], torch.ones_like(Y[1])) and torch.allclose(Y[2], torch.full_like(Y[2], 1e-27), rtol=1e-6, atol=0)
    assert torch.isnan(Y[3]).all() and torch.isnan(Y[4, 6]) and (Y[4, :6] == 0).all() and rstd[4] == 0
    assert (scales[3] == 255).all() and scales[4, 0] == 255 and (scales[4, 1:] == 0).all()
    assert torch.allclose(Y[5], torch.ones_like(Y[5]))


def test_no_rows():
    X, gamma = torch.empty(0, 8, device="cuda"), torch.ones(8, device="cuda")
    maxk.maxk_rms_norm(X, gamma, X.clone())
    dgamma = torch.full((8,), 7.0, device="cuda")
    maxk.maxk_rms_norm_grad(X, X, gamma, torch.empty(0, device="cuda"), X.clone(), dgamma)
    assert (dgamma == 0).all()
