"""Widths past what the microscaled calls take, past 32 bits among them: refused as unsupported, never cut to the bits that an int holds."""
import pytest
import torch

import paper_2312_08656_amd as maxk
from paper_2312_08656_amd import binding

WIDE = (65537, 2 ** 31, 2 ** 32 + 32, 2 ** 40 + 8)  # the last two are 32 and 8 in 32 bits


def _refused(call):
    with pytest.raises(maxk.MaxKError, match="status -2"):
        call()


def _empty(rows, cols, dtype, device):
    return torch.empty((rows, cols), dtype=dtype, device=device)


def _wide_calls(wide, device, rows=4):
    """Calls of `rows` rows with one width past the limit; the tensors fit each other otherwise."""
    f32, u8 = torch.float32, torch.uint8
    t = lambda r, c, dtype=f32: _empty(r, c, dtype, device)
    stored = lambda r, c, bits=4: maxk.mx_empty(r, c, bits, device)
    return {
        "quantize": lambda: maxk.maxk_mx_quantize(t(rows, wide), *stored(rows, wide, 8)),
        "dequantize": lambda: maxk.maxk_mx_dequantize(*stored(rows, wide), t(rows, wide, torch.bfloat16)),
        "linear, columns of Y": lambda: maxk.maxk_mx_linear(*stored(rows, 8), *stored(wide, 8), t(rows, wide)),
        "linear, columns of X": lambda: maxk.maxk_mx_linear(*stored(rows, wide), *stored(8, wide), t(rows, 8)),
        "weight gradient, columns of X": lambda: maxk.maxk_mx_weight_grad(*stored(rows, wide), t(rows, 8), t(8, wide)),
        "weight gradient, columns of dH": lambda: maxk.maxk_mx_weight_grad(*stored(rows, 8), t(rows, wide), t(wide, 8)),
        "weight gradient, k": lambda: maxk.maxk_mx_weight_grad_cbsr(*stored(rows, 8), t(rows, wide), t(rows, wide, u8), t(16, 8)),
        "weight gradient, rows of dW": lambda: maxk.maxk_mx_weight_grad_cbsr(*stored(rows, 8), t(rows, 4), t(rows, 4, torch.int32), t(wide, 8)),
        "input gradient, columns of dX": lambda: maxk.maxk_mx_input_grad(t(rows, 8), *stored(8, wide), t(rows, wide)),
        "input gradient, columns of dH": lambda: maxk.maxk_mx_input_grad(t(rows, wide), *stored(wide, 8), t(rows, 8)),
        "input gradient, k": lambda: maxk.maxk_mx_input_grad_cbsr(t(rows, wide), t(rows, wide, u8), *stored(16, 8), t(rows, 8)),
        "input gradient, rows of W": lambda: maxk.maxk_mx_input_grad_cbsr(t(rows, 4), t(rows, 4, torch.int32), *stored(wide, 8), t(rows, 8)),
    }


@pytest.mark.parametrize("wide", WIDE)
def test_wide_matrices_are_refused(wide):
    for name, call in _wide_calls(wide, "meta").items():  # (shapes alone: 4 rows of 2^40 columns fit no memory)
        try:
            _refused(call)
        except BaseException as e:
            raise AssertionError(name) from e
    _refused(lambda: maxk.mx_weight_grad_workspace(4, wide, 8))
    _refused(lambda: maxk.mx_weight_grad_workspace(4, 8, wide))


def test_the_widest_is_taken():
    widest = 65536
    assert maxk.mx_weight_grad_workspace(4, widest, 8) > 0
    with pytest.raises(maxk.MaxKError, match="device tensor"):  # what is left to refuse
        maxk.maxk_mx_quantize(torch.empty(4, widest), *maxk.mx_empty(4, widest, 8, "cpu"))
    with pytest.raises(maxk.MaxKError, match="device tensor"):
        maxk.maxk_mx_linear(*maxk.mx_empty(4, widest, 4, "meta"), *maxk.mx_empty(8, widest, 4, "meta"), torch.empty(4, 8))


@pytest.mark.gpu
@pytest.mark.parametrize("fast", [True, False])
@pytest.mark.parametrize("wide", WIDE)
def test_wide_device_matrices_are_refused(wide, fast, monkeypatch):
    # matrices without rows: nothing is read or written whatever a call makes of their widths
    binding.load_library()
    if not fast:
        monkeypatch.setattr(binding, "_FAST", None)
    calls = _wide_calls(wide, "cuda", rows=0)
    for name in ("quantize", "dequantize", "weight gradient, k", "input gradient, k"):
        _refused(calls[name])
    few = maxk.mx_empty(0, 8, 4)
    if wide == 65537:
        for name, call in calls.items():
            _refused(call)
        maxk.maxk_mx_quantize(torch.empty(0, 65536, device="cuda"), *maxk.mx_empty(0, 65536, 4))
        maxk.maxk_mx_linear(*few, *maxk.mx_empty(65536, 8, 4), torch.empty(0, 65536, device="cuda"))
