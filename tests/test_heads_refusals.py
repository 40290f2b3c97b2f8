"""What the norm, the log probabilities, distillation and the product of few rows refuse, before anything touches the device."""
import ctypes

import pytest
import torch

import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import binding, build

INVALID, UNSUPPORTED, TOO_SMALL = -1, -2, -5
p, odd, half = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1008)  # never dereferenced
other = ctypes.c_void_p(0x9000)


@pytest.fixture(scope="module")
def lib():
    if not binding.lib_path().exists():
        build.build()
    return binding.load_library()


def each(call, good, changes, status):
    for at, value in changes:
        bad = list(good)
        bad[at] = value
        assert call(*bad, None) == status, (at, value)


NAN, INF = float("nan"), float("inf")


def test_norm(lib):
    #       X, residual, type, N, dim, gamma, eps, H, Y, format, codes, scales, rstd
    good = [p, p, 0, 4, 8, p, 1e-6, p, other, 0, p, p, p]
    each(lib.maxk_rms_norm, good, [(0, None), (1, None), (7, None), (5, None), (10, None), (11, None), (2, 3), (2, -1), (3, -1), (3, 2 ** 31 - 15), (4, 0), (6, 0.0),
                                   (6, -1.0), (6, NAN), (6, INF), (9, 2), (0, odd), (1, odd), (5, odd), (7, odd), (8, odd), (8, p), (10, half), (12, odd)], INVALID)
    each(lib.maxk_rms_norm, good, [(4, maxk.heads._NORM_MAX_DIM + 1)], UNSUPPORTED)
    assert lib.maxk_rms_norm(p, None, 0, 4, 8, p, 1e-6, None, None, 0, None, None, p, None) == INVALID  # nothing to write
    assert lib.maxk_rms_norm(None, None, 0, 0, 8, None, 1e-6, None, None, 0, None, None, None, None) == 0


def test_norm_grad(lib):
    need = lib.maxk_rms_norm_grad_workspace(4, 8)
    assert need > 0 and lib.maxk_rms_norm_grad_workspace(0, 8) > 0
    assert lib.maxk_rms_norm_grad_workspace(-1, 8) == INVALID and lib.maxk_rms_norm_grad_workspace(4, 0) == INVALID
    assert lib.maxk_rms_norm_grad_workspace(4, 16385) == UNSUPPORTED
    #       dY, H, dH, type, N, dim, gamma, rstd, dX, dgamma, workspace, bytes
    good = [p, p, p, 0, 4, 8, p, p, p, p, p, need]
    each(lib.maxk_rms_norm_grad, good, [(0, None), (1, None), (6, None), (7, None), (8, None), (10, None), (3, 3), (4, -1), (5, 0), (0, odd), (1, odd), (2, odd),
                                        (6, odd), (7, odd), (8, odd), (9, odd), (10, half)], INVALID)
    each(lib.maxk_rms_norm_grad, good, [(5, 16385)], UNSUPPORTED)
    each(lib.maxk_rms_norm_grad, good, [(11, need - 1)], TOO_SMALL)


def test_logprobs(lib):
    w = lib.maxk_classes_workspace
    assert w(1000, 100, 5) == 0 and w(1, 100000, 5) > w(1, 100000, 0) > 0
    assert w(-1, 8, 0) == INVALID and w(4, 0, 0) == INVALID and w(4, 8, 9) == INVALID and w(4, 100, 65) == INVALID and w(4, 8, -1) == INVALID
    assert w(4, (1 << 24) + 1, 0) == UNSUPPORTED
    need = w(1, 100000, 5)
    #       logits, type, N, V, labels, label bytes, logprob, entropy, data, index, index bytes, k, workspace, bytes
    good = [p, 0, 1, 100000, p, 8, p, p, p, p, 4, 5, p, need]
    each(lib.maxk_logprobs, good, [(0, None), (4, None), (8, None), (9, None), (12, None), (0, odd), (4, ctypes.c_void_p(0x1004)), (6, odd), (7, odd), (8, odd), (9, odd),
                                   (12, half), (1, 3), (2, -1), (3, 0), (5, 2), (10, 1), (10, 2), (10, 3), (11, 0), (11, -1), (11, 65)], INVALID)
    each(lib.maxk_logprobs, good, [(3, (1 << 24) + 1)], UNSUPPORTED)
    each(lib.maxk_logprobs, good, [(13, need - 1)], TOO_SMALL)
    assert lib.maxk_logprobs(p, 0, 4, 8, p, 8, None, None, None, None, 0, 0, None, 0, None) == INVALID  # nothing to write
    assert lib.maxk_logprobs(None, 0, 0, 8, None, 0, None, None, None, None, 0, 0, None, 0, None) == 0
    need = w(1, 100000, 0)
    #       logits, type, N, V, labels, label bytes, dlogprob, dentropy, logprob, entropy, dlogits, workspace, bytes
    good = [p, 0, 1, 100000, p, 4, p, p, p, p, p, p, need]
    each(lib.maxk_logprobs_grad, good, [(0, None), (4, None), (10, None), (11, None), (0, odd), (4, odd), (6, odd), (7, odd), (8, odd), (9, odd), (10, odd), (1, -1),
                                        (2, -1), (3, 0), (5, 1)], INVALID)
    each(lib.maxk_logprobs_grad, good, [(12, need - 1)], TOO_SMALL)
    assert lib.maxk_logprobs_grad(p, 0, 4, 8, p, 8, None, None, p, p, p, None, 0, None) == INVALID  # no gradient arrives


def test_distill(lib):
    need = lib.maxk_classes_workspace(1, 100000, 0)
    #       logits, type, N, V, data, type, index, index bytes, k, temperature, loss, workspace, bytes
    good = [p, 0, 1, 100000, p, 1, p, 4, 5, 2.0, p, p, need]
    each(lib.maxk_distill, good, [(0, None), (4, None), (6, None), (10, None), (11, None), (0, odd), (4, odd), (6, odd), (10, odd), (11, half), (1, 3), (5, 3), (2, -1), (3, 0), (7, 1),
                                  (7, 2), (7, 0), (8, 0), (9, 0.0), (9, -1.0), (9, NAN), (9, INF), (9, 1e-40), (9, 1e300)], INVALID)
    each(lib.maxk_distill, good, [(3, (1 << 24) + 1), (8, 1025)], UNSUPPORTED)
    each(lib.maxk_distill, good, [(12, need - 1)], TOO_SMALL)
    #       ..., temperature, dloss, loss, dlogits, workspace, bytes
    good = good[:10] + [p, p, p, p, need]
    each(lib.maxk_distill_grad, good, [(10, None), (12, None), (13, None), (10, odd), (11, odd), (12, odd), (8, 0), (9, 0.0)], INVALID)
    each(lib.maxk_distill_grad, good, [(14, need - 1)], TOO_SMALL)
    assert lib.maxk_distill(None, 0, 0, 8, None, 0, None, 1, 5, 1.0, None, None, 0, None) == 0


def test_matvec(lib):
    #       X, type, N, codes, scales, din, dout, bias, Y, type
    good = [p, 0, 4, p, p, 8, 8, p, p, 0]
    each(lib.maxk_mx_matvec, good, [(0, None), (3, None), (4, None), (8, None), (0, odd), (3, half), (7, odd), (8, odd), (1, 3), (9, 3), (9, -1), (2, -1), (5, 0), (6, 0)], INVALID)
    each(lib.maxk_mx_matvec, good, [(5, 65537), (6, (1 << 24) + 1), (2, 1025)], UNSUPPORTED)
    assert lib.maxk_mx_matvec(None, 0, 0, None, None, 8, 8, None, None, 0, None) == 0


def test_the_binding_names_what_does_not_fit(lib):
    X, v8, v4 = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4)
    c8, c4, s = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)
    y, top, idx = torch.zeros(4, dtype=torch.int64), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32)
    w4, ws = torch.zeros(5, 16, dtype=torch.uint8), torch.zeros(5, 1, dtype=torch.uint8)
    r, rg, l, lg, d, dg, m = (maxk.maxk_rms_norm, maxk.maxk_rms_norm_grad, maxk.maxk_logprobs, maxk.maxk_logprobs_grad, maxk.maxk_distill, maxk.maxk_distill_grad,
                              maxk.maxk_mx_matvec)
    refused = {
        "device tensor": [lambda: r(X, v8, X), lambda: rg(X, X, v8, v4, X), lambda: l(X, y, v4), lambda: lg(X, X, y, v4), lambda: d(X, top, idx, v4),
                          lambda: dg(X, top, idx, v4, X), lambda: m(X, w4, ws, torch.zeros(4, 5))],
        "go together": [lambda: r(X, v8), lambda: r(X, v8, X, residual=X), lambda: r(X, v8, X, H=X), lambda: r(X, v8, codes=c8), lambda: r(X, v8, X, scales=s),
                        lambda: l(X, y), lambda: l(X, None, v4), lambda: l(X, y, v4, None, top), lambda: l(X, y, v4, None, None, idx)],
        "codes": [lambda: r(X, v8, codes=c8[:3], scales=s), lambda: r(X, v8, codes=c4.float(), scales=s), lambda: m(X, w4.view(torch.int8), ws, torch.zeros(4, 5)),
                  lambda: m(X, w4[:4], ws, torch.zeros(4, 5))],
        "expected": [lambda: r(X[0], v8, X[0]), lambda: l(X[0], y, v4), lambda: m(X[0], w4, ws, X)],
        "must be [N, k]": [lambda: l(X, y, v4, None, top, idx.long()), lambda: l(X, y, v4, None, top, idx[:, :1]), lambda: l(X, y, v4, None, top[:3], idx[:3]),
                           lambda: d(X, top, idx[:3], v4), lambda: d(X, top[0], idx[0], v4)],
        "k must be": [lambda: l(X, y, v4, None, top[:, :0], idx[:, :0])],
        "labels must be": [lambda: l(X, y.float(), v4), lambda: l(X, y[:3], v4), lambda: lg(X, X, y.short(), v4)],
        "must be given": [lambda: lg(X, X, y), lambda: lg(X, X, None, v4), lambda: lg(X, X, None, None, v4, v4)],
        "Y must be": [lambda: m(X, w4, ws, torch.zeros(3, 5)), lambda: m(X, w4, ws, v8)],
        "bias": [lambda: m(X, w4, ws, torch.zeros(4, 5), v8)],
        "unsupported": [lambda: maxk.rms_norm_grad_workspace(4, 20000), lambda: maxk.classes_workspace(4, 1 << 25), lambda: maxk.classes_workspace(4, 1 << 33),
                        lambda: r(X.new_zeros(1, 20000), v8, X), lambda: l(X.new_zeros(0, 1 << 25), y, v4)],
        "invalid": [lambda: maxk.classes_workspace(4, 100, 65), lambda: maxk.classes_workspace(4, 100, 1 << 40)],
    }
    for word, calls in refused.items():
        for i, call in enumerate(calls):
            with pytest.raises(maxk.MaxKError) as e:
                call()
                pytest.fail(f"{word}: call {i} was made")
            assert word in str(e.value), (word, i, str(e.value))
