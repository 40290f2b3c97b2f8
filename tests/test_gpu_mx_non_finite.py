"""Non-finite values in the operands of the microscaled calls: what a dense product would lose is lost, and nothing else."""
import numpy as np
import pytest
import torch

import mx_common as mx
import paper_2312_08656_amd as maxk
from test_gpu_mx import dev, stored

pytestmark = pytest.mark.gpu

N, DIN, DOUT, K = 70, 96, 80, 9


def _lost(t):
    return ~torch.isfinite(t).cpu().numpy()


def _gradient(rng, kind):
    """(the call's tensors, those of row 3, column) of one entry of the gradient: a dense one in each type, or CBSR."""
    dH = rng.standard_normal((N, DOUT)).astype(np.float32)
    if kind != "cbsr":
        t = dev(dH).to(getattr(torch, kind))
        return (t,), t[3], 11, 11
    cols = mx.columns(rng, N, DOUT, K)
    values = dev(np.take_along_axis(dH, cols, 1))
    return (values, dev(cols.astype(np.uint8))), values[3], 4, int(cols[3, 4])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16", "cbsr"])
def test_a_value_of_the_gradient(kind, value):
    rng = np.random.default_rng(91)
    given, row, at, column = _gradient(rng, kind)
    row[at] = value
    c, s = stored(mx.features(rng, N, DIN) + 0.1, 8)[2:]
    wc, ws = stored(mx.features(rng, DOUT, DIN, 0.3), 4)[2:]
    dW, db, dX = torch.zeros(DOUT, DIN, device="cuda"), torch.zeros(DOUT, device="cuda"), torch.zeros(N, DIN, device="cuda")
    (maxk.maxk_mx_weight_grad_cbsr if kind == "cbsr" else maxk.maxk_mx_weight_grad)(c, s, *given, dW, db)
    (maxk.maxk_mx_input_grad_cbsr if kind == "cbsr" else maxk.maxk_mx_input_grad)(*given, wc, ws, dX)
    for got, lost in ((dW, column), (db, column), (dX, 3)):  # a row of dW, an entry of db, a row of dX: all of it, and no other
        bad = _lost(got).reshape(got.shape[0], -1)
        assert bad[lost].all() and not np.delete(bad, lost, axis=0).any()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16", "cbsr"])
def test_a_block_of_a_checkpoint_and_of_the_weights(kind, bits):
    rng = np.random.default_rng(92)
    given = _gradient(rng, kind)[0]
    X, W = mx.features(rng, N, DIN), mx.features(rng, DOUT, DIN, 0.3)
    X[7, 40], W[20, 70] = np.inf, np.nan
    dW, db, dX = torch.zeros(DOUT, DIN, device="cuda"), torch.zeros(DOUT, device="cuda"), torch.zeros(N, DIN, device="cuda")
    (maxk.maxk_mx_weight_grad_cbsr if kind == "cbsr" else maxk.maxk_mx_weight_grad)(*stored(X, bits)[2:], *given, dW, db)
    (maxk.maxk_mx_input_grad_cbsr if kind == "cbsr" else maxk.maxk_mx_input_grad)(*given, *stored(W, 4)[2:], dX)
    bad = _lost(dW)
    assert bad[:, 32:64].all() and not bad[:, :32].any() and not bad[:, 64:].any() and not _lost(db).any()
    bad = _lost(dX)
    assert bad[:, 64:].all() and not bad[:, :64].any()


def test_a_block_of_either_operand_of_the_product():
    rng = np.random.default_rng(93)
    X, W = mx.features(rng, N, DIN), mx.features(rng, DOUT, DIN, 0.3)
    X[7, 95], W[20, 0] = np.nan, -np.inf
    Y = torch.zeros(N, DOUT, device="cuda")
    maxk.maxk_mx_linear(*stored(X, 4)[2:], *stored(W, 4)[2:], Y)
    bad = _lost(Y)
    assert bad[7].all() and bad[:, 20].all() and not np.delete(np.delete(bad, 7, 0), 20, 1).any()
