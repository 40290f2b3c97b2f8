"""Gradients of the microscaled calls for operands near either end of what fp32 and the scale byte hold."""
import numpy as np
import pytest
import torch

import mx_common as mx
import paper_2312_08656_amd as maxk
from test_gpu_mx import dev, host, stored

pytestmark = pytest.mark.gpu

N, DIN, DOUT, K = 300, 96, 80, 8
LEAST = 2.0 ** -126  # least normal number


def _bound(D, X, n, parts):
    """As where nothing is small, 8 + sqrt(terms) units of 2^-24 of the sum of |terms|; a part or an operand below the normal numbers counts as the least
    of them, as the matrix unit lines products up by their exponents.  Of an fp32 gradient (3 parts) what lies below 2^-133 is dropped; sums round to 2^-149."""
    there = (D != 0).astype(np.float64)
    terms = (np.abs(D) + parts * LEAST * there) @ (np.abs(X) + LEAST)
    dropped = 2.0 ** -133 * there @ np.abs(X) if parts == 3 else 0.0
    return (8 + np.sqrt(parts * n)) * 2.0 ** -24 * terms + dropped + n * 2.0 ** -149


# exponents of dH and of the other operand
SIZES = [(-100, 100), (-116, 110), (-124, 115), (-130, 110), (-125, 0), (-148, 120), (100, -100), (110, -126), (110, -130), (120, -80), (118, -100), (-60, 120), (-60, -50), (0, -125)]


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "cbsr"])
@pytest.mark.parametrize("small,large", SIZES)
def test_gradients_of_extreme_sizes(small, large, kind):
    rng = np.random.default_rng(1000 - small + large)
    dH = np.ldexp(np.clip(rng.standard_normal((N, DOUT)), -3.9, 3.9), small).astype(np.float32)
    if kind == "cbsr":
        cols = mx.columns(rng, N, DOUT, K)
        dXs = np.take_along_axis(dH, cols, 1)
        given, D = (dev(dXs), dev(cols.astype(np.uint8))), mx.scatter(dXs, cols, DOUT)
    else:
        given = (dev(dH).to(getattr(torch, kind)),)
        D = given[0].double().cpu().numpy()
    parts = 1 if kind == "bfloat16" else 3
    for bits in (8, 4):
        codes, scales, c, s = stored(np.ldexp(mx.features(rng, N, DIN, 0.3), large).astype(np.float32), bits)
        X = mx.values(codes, scales, DIN)
        dW, db = torch.empty(DOUT, DIN, device="cuda"), torch.empty(DOUT, device="cuda")
        (maxk.maxk_mx_weight_grad_cbsr if kind == "cbsr" else maxk.maxk_mx_weight_grad)(c, s, *given, dW, db)
        assert (np.abs(host(dW) - D.T @ X) <= _bound(D.T, X, N, parts)).all()
        ones = np.ones((N, 1))
        assert (np.abs(host(db) - D.sum(axis=0)) <= _bound(D.T, ones, N, parts)[:, 0]).all()
    codes, scales, c, s = stored(np.ldexp(mx.features(rng, DOUT, DIN, 0.3), large).astype(np.float32), 4)
    W = mx.values(codes, scales, DIN)
    dX = torch.empty(N, DIN, device="cuda")
    (maxk.maxk_mx_input_grad_cbsr if kind == "cbsr" else maxk.maxk_mx_input_grad)(*given, c, s, dX)
    assert (np.abs(host(dX) - D @ W) <= _bound(D, W, K if kind == "cbsr" else DOUT, parts)).all()


def test_the_largest_gradients_keep_their_bits():
    # one value a row against whole numbers: the products are exact, and only a part that is lost would show
    rng = np.random.default_rng(210)
    X = rng.integers(-1, 2, (DOUT, DIN)).astype(np.float32)
    c, s = stored(X, 4)[2:]
    values = np.concatenate([np.nextafter(np.float32(2.0) ** e, np.float32(np.inf), dtype=np.float32) * np.ones(1, np.float32) for e in range(-109, 127)] +
                            [np.array([np.finfo(np.float32).max, -np.finfo(np.float32).max, 1 / 3, -2.0 ** 127 * 1.9999998], np.float32)])
    dH = np.zeros((len(values), DOUT), np.float32)
    at = rng.integers(0, DOUT, len(values))
    dH[np.arange(len(values)), at] = values
    dX = torch.empty(len(values), DIN, device="cuda")
    maxk.maxk_mx_input_grad(dev(dH), c, s, dX)
    np.testing.assert_array_equal(host(dX), values.astype(np.float64)[:, None] * X[at])
