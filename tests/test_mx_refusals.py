"""What the microscaled calls refuse, before anything touches the device."""
import ctypes

import pytest
import torch

import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import binding, build

INVALID, UNSUPPORTED, TOO_SMALL = -1, -2, -5


@pytest.fixture(scope="module")
def lib():
    if not binding.lib_path().exists():
        build.build()
    return binding.load_library()


def test_c_calls_check_their_arguments(lib):
    p, odd, half = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1008)  # never dereferenced
    q, d, l = lib.maxk_mx_quantize, lib.maxk_mx_dequantize, lib.maxk_mx_linear
    for bad in ((p, 3, 4, 8, 0, p, p), (p, -1, 4, 8, 0, p, p), (p, 0, -1, 8, 0, p, p), (p, 0, 4, 0, 0, p, p), (p, 0, 4, 8, 2, p, p), (p, 0, 4, 8, -1, p, p),
                (None, 0, 4, 8, 0, p, p), (p, 0, 4, 8, 0, None, p), (p, 0, 4, 8, 0, p, None), (odd, 0, 4, 8, 0, p, p), (odd, 1, 4, 8, 0, p, p),
                (p, 0, 4, 8, 0, half, p), (p, 0, 2 ** 31 - 15, 8, 0, p, p)):
        assert q(*bad, None) == INVALID, bad
        X, vt, N, din, fmt, codes, scales = bad
        assert d(codes, scales, fmt, N, din, X, vt, None) == INVALID, bad
    assert q(p, 0, 4, 65537, 0, p, p, None) == UNSUPPORTED and d(p, p, 0, 4, 65537, p, 0, None) == UNSUPPORTED
    assert q(None, 0, 0, 8, 0, None, None, None) == 0 and d(None, None, 0, 0, 8, None, 0, None) == 0
    good = [p, p, 4, p, p, 8, 8, p, p, 0]
    for at, value in ((0, None), (1, None), (3, None), (4, None), (8, None), (0, half), (3, half), (7, odd), (8, odd), (2, -1), (5, 0), (6, 0), (9, 3)):
        bad = list(good)
        bad[at] = value
        assert l(*bad, None) == INVALID, (at, value)
    assert l(*[p, p, 4, p, p, 8, 65537, p, p, 0], None) == UNSUPPORTED
    assert l(None, None, 0, None, None, 8, 8, None, None, 0, None) == 0


def test_c_gradient_calls_check_their_arguments(lib):
    p, odd, half = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1008)
    need = lib.maxk_mx_weight_grad_workspace(4, 8, 8)
    assert need > 0 and lib.maxk_mx_weight_grad_workspace(0, 8, 8) > 0
    assert lib.maxk_mx_weight_grad_workspace(-1, 8, 8) == INVALID and lib.maxk_mx_weight_grad_workspace(4, 0, 8) == INVALID
    assert lib.maxk_mx_weight_grad_workspace(4, 8, 65537) == UNSUPPORTED
    good = [p, p, 0, 4, 8, 8, p, 0, p, p, p, need]
    for at, value in ((0, None), (1, None), (6, None), (8, None), (10, None), (0, half), (6, odd), (8, odd), (9, odd), (10, half), (2, 2), (3, -1), (4, 0),
                      (5, 0), (7, 3)):
        bad = list(good)
        bad[at] = value
        assert lib.maxk_mx_weight_grad(*bad, None) == INVALID, (at, value)
    assert lib.maxk_mx_weight_grad(*good[:-1], need - 1, None) == TOO_SMALL
    good = [p, p, 0, 4, 8, 8, p, p, 1, 2, p, p, p, need]
    for at, value in ((6, None), (7, None), (6, odd), (8, 3), (8, 0), (9, 0), (9, 9), (12, None), (5, 1)):
        bad = list(good)
        bad[at] = value
        assert lib.maxk_mx_weight_grad_cbsr(*bad, None) == INVALID, (at, value)
    assert lib.maxk_mx_weight_grad_cbsr(p, p, 0, 4, 8, 257, p, p, 1, 2, p, p, p, 1 << 30, None) == INVALID  # columns past a byte
    assert lib.maxk_mx_weight_grad_cbsr(p, p, 0, 4, 8, 257, p, odd, 2, 2, p, p, p, 1 << 30, None) == INVALID
    good = [p, 0, 4, p, p, 8, 8, p, 0]
    for at, value in ((0, None), (3, None), (4, None), (7, None), (0, odd), (3, half), (7, odd), (1, 3), (2, -1), (5, 0), (6, 0), (8, -1)):
        bad = list(good)
        bad[at] = value
        assert lib.maxk_mx_input_grad(*bad, None) == INVALID, (at, value)
    good = [p, p, 1, 2, 4, p, p, 8, 8, p, 0]
    for at, value in ((0, None), (1, None), (2, 3), (3, 0), (3, 9), (9, None), (0, odd)):
        bad = list(good)
        bad[at] = value
        assert lib.maxk_mx_input_grad_cbsr(*bad, None) == INVALID, (at, value)
    assert lib.maxk_mx_input_grad_cbsr(p, p, 1, 2, 4, p, p, 65537, 8, p, 0, None) == UNSUPPORTED
    assert lib.maxk_mx_input_grad(None, 0, 0, None, None, 8, 8, None, 0, None) == 0


def test_the_binding_names_what_does_not_fit(lib):
    X = torch.zeros(4, 40)
    c8, c4, s = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    dH, dW, dXs, idx = torch.zeros(4, 8), torch.zeros(8, 40), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.uint8)
    w4, ws = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.uint8)
    refused = [
        lambda: maxk.maxk_mx_quantize(X, c8, s),  # host tensors
        lambda: maxk.maxk_mx_quantize(X, c8.float(), s),
        lambda: maxk.maxk_mx_quantize(X, c8[:, :40], s),
        lambda: maxk.maxk_mx_quantize(X, c8, s[:3]),
        lambda: maxk.maxk_mx_quantize(X[0], c8, s),
        lambda: maxk.maxk_mx_quantize(X.double(), c8, s),
        lambda: maxk.maxk_mx_dequantize(c4, s, X),
        lambda: maxk.maxk_mx_dequantize(c4, s, torch.zeros(4, 65)),
        lambda: maxk.maxk_mx_linear(c8, s, w4, ws, dH),  # 8 bits
        lambda: maxk.maxk_mx_linear(c4, s, w4[:, :16], ws[:, :1], dH),  # other width
        lambda: maxk.maxk_mx_linear(c4, s, w4, ws, torch.zeros(4, 9)),
        lambda: maxk.maxk_mx_linear(c4, s, w4, ws, dH, torch.zeros(9)),
        lambda: maxk.maxk_mx_weight_grad(c8, s, dH, dW),
        lambda: maxk.maxk_mx_weight_grad(c8, s, dH[:3], dW),
        lambda: maxk.maxk_mx_weight_grad(c8, s, dH, dW.t()),
        lambda: maxk.maxk_mx_weight_grad(c8, s, dH, dW, torch.zeros(7)),
        lambda: maxk.maxk_mx_weight_grad_cbsr(c8, s, dXs, idx[:, :1], dW),
        lambda: maxk.maxk_mx_weight_grad_cbsr(c8, s, dXs, idx.long(), dW),
        lambda: maxk.maxk_mx_input_grad(dH, w4, ws, X),
        lambda: maxk.maxk_mx_input_grad(dH, w4, ws, X[:3]),
        lambda: maxk.maxk_mx_input_grad_cbsr(dXs, idx, w4, ws[:, :1], X),
        lambda: maxk.mx_empty(4, 8, 5, device="cpu"),
        lambda: maxk.mx_weight_grad_workspace(4, 70000, 8),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(maxk.MaxKError):
            call()
            pytest.fail(f"call {i} was made")
