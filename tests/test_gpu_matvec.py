"""Products of few unrounded rows with 4-bit weights against 64 bits."""
import numpy as np
import pytest
import torch

import heads_common as hc
import mx_common
import paper_2312_08656_amd as maxk

pytestmark = pytest.mark.gpu


def weights(rng, dout, din):
    W = mx_common.features(rng, dout, din) / np.sqrt(din)
    codes, scales = mx_common.quantize(W, 4)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), mx_common.values(codes, scales, din)


def check(X, codes, scales, W, bias, y_dtype):
    N, dout = X.shape[0], W.shape[0]
    Y = torch.full((N, dout), 7, dtype=y_dtype, device="cuda")
    maxk.maxk_mx_matvec(X, codes, scales, Y, bias)
    x = hc.f64(X)
    want, size = x @ W.T, np.abs(x) @ np.abs(W).T
    if bias is not None:
        want, size = want + hc.f64(bias), size + np.abs(hc.f64(bias))
    # products are exact, up to three parts each; sums of them in any order: the root of their number, as everywhere on matrix instructions
    hc.close(Y, want, (8 + np.sqrt(3 * x.shape[1])) * hc.U * size, y_dtype)
    return Y


@pytest.mark.parametrize("dtype", hc.TYPES, ids=str)
@pytest.mark.parametrize("N", [1, 2, 5, 16, 17, 40])
@pytest.mark.parametrize("din,dout", [(1, 1), (31, 17), (32, 16), (100, 47), (256, 256), (500, 33), (512, 64), (513, 15), (1433, 100), (4096, 65), (9000, 31), (16000, 20), (33000, 9), (65536, 5)])
def test_matvec(din, dout, N, dtype):
    rng = np.random.default_rng(din + N)
    codes, scales, W = weights(rng, dout, din)
    X = torch.from_numpy(mx_common.features(rng, N, din)).cuda().to(dtype)
    bias = torch.from_numpy(rng.standard_normal(dout).astype(np.float32)).cuda()
    for y_dtype in {torch.float32, dtype}:
        check(X, codes, scales, W, bias, y_dtype)
    check(X, codes, scales, W, None, torch.bfloat16)


@pytest.mark.parametrize("N", [1, 3, 9, 16])
def test_many_rows_of_weights(N):
    rng = np.random.default_rng(N)
    codes, scales, W = weights(rng, 20011, 200)
    for dtype in hc.TYPES:
        check(torch.from_numpy(mx_common.features(rng, N, 200)).cuda().to(dtype), codes, scales, W, None, dtype)


@pytest.mark.parametrize("din,dout", [(1100, 33001), (9001, 6500), (4096, 6200), (2049, 32800)])
def test_many_columns_and_rows(din, dout):
    """Two tiles a wavefront, few and many wavefronts, several rounds of each, the last one whole and not."""
    rng = np.random.default_rng(din)
    codes, scales, W = weights(rng, dout, din)
    for N, dtype in ((3, torch.float32), (16, torch.bfloat16), (5, torch.float16), (2, torch.bfloat16)):
        check(torch.from_numpy(mx_common.features(rng, N, din)).cuda().to(dtype), codes, scales, W, None, dtype)


def test_most_rows():
    rng = np.random.default_rng(9)
    codes, scales, W = weights(rng, 300, 1030)
    for N, dtype in ((1024, torch.float32), (1000, torch.bfloat16), (129, torch.float16)):
        check(torch.from_numpy(mx_common.features(rng, N, 1030)).cuda().to(dtype), codes, scales, W, None, dtype)


def test_more_workgroups_than_a_launch_of_one_dimension_has():
    """A row of X by four rows of W a workgroup of 1024 threads: 2^22 rows are 2^30 threads, past them the grid's second dimension begins; codes and offsets past 2^32 bytes."""
    din, dout = 16416, (1 << 22) + 5
    codes, scales = torch.zeros(dout, din // 2, dtype=torch.uint8, device="cuda"), torch.full((dout, din // 32), 127, dtype=torch.uint8, device="cuda")
    some = [0, 3, (1 << 20) + 1, (1 << 22) - 1, 1 << 22, dout - 1]
    for i, o in enumerate(some):
        codes[o, 1000 + i] = 0x2A  # the even column -1, the odd one 1
        codes[o, din // 2 - 1] = 0x60  # the last column 4
    X = torch.arange(din, device="cuda", dtype=torch.float32).view(1, din)
    Y = torch.full((1, dout), 7.0, device="cuda")
    maxk.maxk_mx_matvec(X, codes, scales, Y)
    assert torch.equal(Y[0, some], torch.full((len(some),), 1.0 + 4 * (din - 1), device="cuda"))
    Y[0, some] = 0
    assert not Y.any()


def test_offsets_and_what_lies_around():
    rng = np.random.default_rng(4)
    N, din, dout = 3, 77, 45
    codes, scales, W = weights(rng, dout, din)
    X = torch.from_numpy(mx_common.features(rng, N, din)).cuda()
    for dtype in hc.TYPES:
        want = check(X.to(dtype), codes, scales, W, None, dtype)
        for at in (1, 2, 3):
            flat = torch.full((N * din + 8,), float("nan"), dtype=dtype, device="cuda")
            flat[at:at + N * din] = X.to(dtype).view(-1)
            out = torch.full((N * dout + 8,), 3.0, dtype=dtype, device="cuda")
            maxk.maxk_mx_matvec(flat[at:at + N * din].view(N, din), codes, scales, out[at:at + N * dout].view(N, dout))
            assert torch.equal(out[at:at + N * dout].view(N, dout), want) and (out[:at] == 3).all() and (out[at + N * dout:] == 3).all()


def test_extremes_and_non_finite():
    din, dout = 64, 20
    W = np.zeros((dout, din), dtype=np.float32)
    W[:, 3] = np.ldexp(1.0, np.arange(dout) * 10 - 100)
    codes, scales = mx_common.quantize(W, 4)
    codes, scales = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    X = torch.zeros(4, din, device="cuda")
    X[0, 3] = 1.5e-30
    X[1, 3] = float("inf")
    X[2, 40] = float("nan")
    Y = torch.empty(4, dout, device="cuda")
    maxk.maxk_mx_matvec(X, codes, scales, Y)
    want = np.float64(np.float32(1.5e-30)) * W[:, 3].astype(np.float64)
    # smaller sums may be flushed to 0, and each of the three parts' products is rounded to the step of fp32 there, 2^-149: 1.5 steps in all
    keep = np.abs(want) >= 2.0 ** -126
    assert np.array_equal(hc.f64(Y[0])[keep], want.astype(np.float32)[keep]) and (hc.f64(Y[0])[~keep] <= want[~keep] + 1.5 * 2.0 ** -149).all()
    assert not torch.isfinite(Y[1]).any() and torch.isnan(Y[2]).all() and (Y[3] == 0).all()
    scales[7, 1] = 255  # a block that stands for NaN
    maxk.maxk_mx_matvec(X, codes, scales, Y)
    assert torch.isnan(Y[3, 7]) and torch.equal(Y[3].isnan().nonzero()[:, 0].cpu(), torch.tensor([7]))


def test_no_rows():
    codes, scales = maxk.mx_empty(5, 40, 4)
    maxk.maxk_mx_matvec(torch.empty(0, 40, device="cuda"), codes, scales, torch.empty(0, 5, device="cuda"))
