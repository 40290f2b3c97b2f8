"""The microscaled operators at widths around and past what one workgroup holds: column groups that do not divide evenly, gradients taken in chunks."""
import numpy as np
import pytest
import torch

import mx_common as mx
import paper_2312_08656_amd as maxk
from test_gpu_mx import check, dev, gradient, host, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dout", [64, 65, 129, 192, 193, 320, 385, 400, 448, 449, 640, 769, 1100])
def test_linear_widths_out(dout):
    rng = np.random.default_rng(dout)
    for N, din in ((1, 40), (37, 200), (100, 64)):
        x_codes, x_scales, xc, xs = stored(mx.features(rng, N, din), 4)
        w_codes, w_scales, wc, ws = stored(mx.features(rng, dout, din, 0.3) / np.sqrt(din), 4)
        X, W = mx.values(x_codes, x_scales, din), mx.values(w_codes, w_scales, din)
        for kind in ("f32", "bf16"):
            Y = torch.full((N, dout), float("nan"), dtype=torch.float32 if kind == "f32" else torch.bfloat16, device="cuda")
            maxk.maxk_mx_linear(xc, xs, wc, ws, Y)
            check(host(Y), X @ W.T, np.abs(X) @ np.abs(W).T, din, kind)


@pytest.mark.parametrize("din", [31, 128, 129, 257, 512, 513, 1024, 1025, 2500])
def test_linear_widths_in(din):
    rng = np.random.default_rng(din)
    x_codes, x_scales, xc, xs = stored(mx.features(rng, 50, din), 4)
    w_codes, w_scales, wc, ws = stored(mx.features(rng, 70, din, 0.3) / np.sqrt(din), 4)
    X, W = mx.values(x_codes, x_scales, din), mx.values(w_codes, w_scales, din)
    Y = torch.full((50, 70), float("nan"), device="cuda")
    maxk.maxk_mx_linear(xc, xs, wc, ws, Y)
    check(host(Y), X @ W.T, np.abs(X) @ np.abs(W).T, din)


@pytest.mark.parametrize("k", [0, 1, 40, 200])
@pytest.mark.parametrize("dout", [200, 255, 257, 384, 512, 516, 700, 1030])
def test_gradients_of_widths_out(dout, k):
    rng = np.random.default_rng(dout + k)
    for N, din, kinds in ((70, 96, ("f32", "bf16", "f16")), (33, 270, ("f32",))):
        codes, scales, c, s = stored(mx.features(rng, N, din), 8)
        w_codes, w_scales, wc, ws = stored(mx.features(rng, dout, din, 0.3) / np.sqrt(din), 4)
        X, W = mx.values(codes, scales, din), mx.values(w_codes, w_scales, din)
        for kind in kinds if k == 0 else ("f32",):
            given, dH = gradient(rng, N, dout, k, kind, np.int16)
            dW, db = torch.full((dout, din), float("nan"), device="cuda"), torch.full((dout,), float("nan"), device="cuda")
            dX = torch.full((N, din), float("nan"), device="cuda")
            (maxk.maxk_mx_weight_grad_cbsr if k else maxk.maxk_mx_weight_grad)(c, s, *given, dW, db)
            (maxk.maxk_mx_input_grad_cbsr if k else maxk.maxk_mx_input_grad)(*given, wc, ws, dX)
            check(host(dW), dH.T @ X, np.abs(dH).T @ np.abs(X), N)
            check(host(db), dH.sum(axis=0), np.abs(dH).sum(axis=0), N)
            check(host(dX), dH @ W, np.abs(dH) @ np.abs(W), dout)


@pytest.mark.parametrize("din", [63, 65, 127, 129, 256, 260, 700, 1500])
def test_gradients_of_widths_in(din):
    rng = np.random.default_rng(din)
    for N, dout, k in ((40, 48, 0), (40, 130, 20), (90, 260, 33)):
        codes, scales, c, s = stored(mx.features(rng, N, din), 4)
        w_codes, w_scales, wc, ws = stored(mx.features(rng, dout, din, 0.3) / np.sqrt(din), 4)
        X, W = mx.values(codes, scales, din), mx.values(w_codes, w_scales, din)
        given, dH = gradient(rng, N, dout, k, "f32", np.int32)
        dW, dX = torch.full((dout, din), float("nan"), device="cuda"), torch.full((N, din), float("nan"), device="cuda")
        (maxk.maxk_mx_weight_grad_cbsr if k else maxk.maxk_mx_weight_grad)(c, s, *given, dW)
        (maxk.maxk_mx_input_grad_cbsr if k else maxk.maxk_mx_input_grad)(*given, wc, ws, dX)
        check(host(dW), dH.T @ X, np.abs(dH).T @ np.abs(X), N)
        check(host(dX), dH @ W, np.abs(dH) @ np.abs(W), dout)


def test_rows_around_the_ranges():
    # row counts at which ranges, rounds and groups come out uneven
    rng = np.random.default_rng(71)
    for din, dout, k in ((64, 64, 8), (100, 100, 13), (64, 256, 32), (130, 300, 0)):
        for N in (31, 32, 33, 63, 65, 127, 129, 255, 257, 511, 513, 1000, 2047, 2049, 4100, 9000):
            codes, scales, c, s = stored(mx.features(rng, N, din), 8)
            X = mx.values(codes, scales, din)
            given, dH = gradient(rng, N, dout, k, "f32", np.int16)
            dW, db = torch.full((dout, din), float("nan"), device="cuda"), torch.full((dout,), float("nan"), device="cuda")
            (maxk.maxk_mx_weight_grad_cbsr if k else maxk.maxk_mx_weight_grad)(c, s, *given, dW, db)
            check(host(dW), dH.T @ X, np.abs(dH).T @ np.abs(X), N)
            check(host(db), dH.sum(axis=0), np.abs(dH).sum(axis=0), N)


def test_a_row_that_is_nan_and_gradients_of_infinity():
    # a NaN block of X: its columns of dW, as in a dense product; a NaN or Inf in dH: its row of dW, its db, its row of dX
    rng = np.random.default_rng(81)
    N, din, dout = 50, 96, 80
    X = mx.features(rng, N, din)
    X[7, 40] = np.inf
    codes, scales, c, s = stored(X, 8)
    wc, ws = stored(mx.features(rng, dout, din, 0.3), 4)[2:]
    dH = rng.standard_normal((N, dout)).astype(np.float32)
    dW, db, dX = torch.empty(dout, din, device="cuda"), torch.empty(dout, device="cuda"), torch.empty(N, din, device="cuda")
    maxk.maxk_mx_weight_grad(c, s, dev(dH), dW, db)
    bad = ~np.isfinite(host(dW))
    assert bad[:, 32:64].all() and not bad[:, :32].any() and not bad[:, 64:].any() and np.isfinite(host(db)).all()
    c, s = stored(mx.features(rng, N, din) + 0.1, 8)[2:]
    for value in (np.nan, np.inf):
        dH[3, 11] = value
        maxk.maxk_mx_weight_grad(c, s, dev(dH), dW, db)
        maxk.maxk_mx_input_grad(dev(dH), wc, ws, dX)
        bad = ~np.isfinite(host(dW))
        assert bad[11].all() and not np.delete(bad, 11, axis=0).any()
        assert not np.isfinite(host(db)[11]) and np.isfinite(np.delete(host(db), 11)).all()
        bad = ~np.isfinite(host(dX))
        assert bad[3].any() and not np.delete(bad, 3, axis=0).any()


@pytest.mark.parametrize("k", [0, 12, 50, 200])
@pytest.mark.parametrize("dout", [200, 257, 384, 516])
def test_weight_gradients_of_many_rows(dout, k):
    # row counts from which tiles of 128 and 256 columns of dH are taken, with widths that do not fill them
    rng = np.random.default_rng(3 * dout + k)
    for N, din, kinds in ((20001, 270, ("f32", "bf16", "f16")), (30070, 100, ("f32",))):
        codes, scales, c, s = stored(mx.features(rng, N, din), 8)
        X = mx.values(codes, scales, din)
        for kind in kinds if k == 0 else ("f32",):
            given, dH = gradient(rng, N, dout, k, kind, np.int16)
            dW, db = torch.full((dout, din), float("nan"), device="cuda"), torch.full((dout,), float("nan"), device="cuda")
            (maxk.maxk_mx_weight_grad_cbsr if k else maxk.maxk_mx_weight_grad)(c, s, *given, dW, db)
            check(host(dW), dH.T @ X, np.abs(dH).T @ np.abs(X), N)
            check(host(db), dH.sum(axis=0), np.abs(dH).sum(axis=0), N)
