"""Microscaled storage and the linear half of a layer on it (see include/maxk.h for formats and the contract of each call).

Codes are int8 [N, 32 nb] (MX8) or uint8 [N, 16 nb] (MX4, two codes a byte), scales uint8 [N, nb], nb = ceil(din / 32): the dtype of the codes
says which format they are.  As in the rest of the binding, outputs are given by the caller and overwritten, and every call enqueues on
the current stream.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as _b
from .binding import MaxKError

MX_8, MX_4 = 0, 1
_MAX_DIM = 65536  # MAXK_MX_MAX_DIM
_MAX_CLASSES = 1 << 24  # MAXK_MAX_CLASSES
_UNSUPPORTED = -2
_FORMAT = {torch.int8: MX_8, torch.uint8: MX_4}


def mx_blocks(din: int) -> int:
    """Blocks of 32 columns in a row of din."""
    return (din + 31) // 32


def mx_empty(N: int, din: int, bits: int, device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
    """(codes, scales) for an [N, din] matrix in 8 or 4 bits, not filled."""
    if bits not in (8, 4):
        raise MaxKError("mx_empty: bits must be 8 or 4")
    nb = mx_blocks(din)
    return (torch.empty((N, nb * (32 if bits == 8 else 16)), dtype=torch.int8 if bits == 8 else torch.uint8, device=device),
            torch.empty((N, nb), dtype=torch.uint8, device=device))


def _stored(codes: torch.Tensor, scales: torch.Tensor, rows: int, din: int, what: str, only4: bool = False) -> int:
    """The format of (codes, scales), which must be [rows, din] in it."""
    fmt = _FORMAT.get(codes.dtype)
    if fmt is None or (only4 and fmt != MX_4):
        raise MaxKError(f"{what}: codes must be " + ("uint8 (4 bits)" if only4 else "int8 (8 bits) or uint8 (4 bits)"))
    nb = mx_blocks(din)
    if tuple(codes.shape) != (rows, nb * (32 if fmt == MX_8 else 16)) or tuple(scales.shape) != (rows, nb):
        raise MaxKError(f"{what}: codes / scales do not fit [{rows}, {din}]")
    return fmt


def _value(t: torch.Tensor, what: str) -> int:
    if t.dtype not in _b._VALUE_TYPE:
        raise MaxKError(f"{what}: expected float32, bfloat16 or float16")
    return _b._VALUE_TYPE[t.dtype]


def _width(n: int, what: str) -> int:
    """n, refused here where the library's 32 bits might not hold it."""
    if n > _MAX_DIM:
        _b._check(_UNSUPPORTED, what)
    return n


def _matrix(t: torch.Tensor, what: str) -> Tuple[int, int]:
    if t.dim() != 2:
        raise MaxKError(f"{what}: expected a matrix")
    return t.shape[0], _width(t.shape[1], what)


def maxk_mx_quantize(X: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor) -> None:
    """codes and scales are overwritten with X [N, din] (float32, bfloat16, float16) in the format of codes."""
    if _b._FAST is not None and _b._FAST.mx_quantize(X, codes, scales):
        return
    N, din = _matrix(X, "maxk_mx_quantize: X")
    fmt = _stored(codes, scales, N, din, "maxk_mx_quantize")
    _b._check(_b.load_library().maxk_mx_quantize(_b._dev(X, X.dtype, "X"), _value(X, "maxk_mx_quantize: X"), N, din, fmt,
                                                 _b._dev(codes, codes.dtype, "codes"), _b._dev(scales, torch.uint8, "scales"), _b._stream()),
              "maxk_mx_quantize")


def maxk_mx_dequantize(codes: torch.Tensor, scales: torch.Tensor, X: torch.Tensor) -> None:
    """X [N, din] (float32, bfloat16, float16) is overwritten with what codes and scales stand for."""
    if _b._FAST is not None and _b._FAST.mx_dequantize(codes, scales, X):
        return
    N, din = _matrix(X, "maxk_mx_dequantize: X")
    fmt = _stored(codes, scales, N, din, "maxk_mx_dequantize")
    _b._check(_b.load_library().maxk_mx_dequantize(_b._dev(codes, codes.dtype, "codes"), _b._dev(scales, torch.uint8, "scales"), fmt, N, din,
                                                   _b._dev(X, X.dtype, "X"), _value(X, "maxk_mx_dequantize: X"), _b._stream()),
              "maxk_mx_dequantize")


def _same_width(a: torch.Tensor, b: torch.Tensor, what: str) -> int:
    """Columns of two 4-bit matrices, rounded up to whole blocks (what lies past din is zero in either)."""
    if _matrix(a, what)[1] != _matrix(b, what)[1]:
        raise MaxKError(f"{what}: the operands' blocks do not match")
    return _width(32 * a.shape[1], what)


def maxk_mx_linear(x_codes: torch.Tensor, x_scales: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, Y: torch.Tensor,
                   bias: Optional[torch.Tensor] = None) -> None:
    """Y [N, dout] (float32, bfloat16, float16) is overwritten with X W^T + bias, X [N, din] and W [dout, din] both in 4 bits."""
    if _b._FAST is not None and _b._FAST.mx_linear(x_codes, x_scales, w_codes, w_scales, Y, bias):
        return
    N, dout = _matrix(Y, "maxk_mx_linear: Y")
    din = _same_width(x_scales, w_scales, "maxk_mx_linear")
    _stored(x_codes, x_scales, N, din, "maxk_mx_linear: X", True)
    _stored(w_codes, w_scales, dout, din, "maxk_mx_linear: W", True)
    if bias is not None and tuple(bias.shape) != (dout,):
        raise MaxKError("maxk_mx_linear: bias must be [dout]")
    _b._check(_b.load_library().maxk_mx_linear(
        _b._dev(x_codes, torch.uint8, "x_codes"), _b._dev(x_scales, torch.uint8, "x_scales"), N, _b._dev(w_codes, torch.uint8, "w_codes"),
        _b._dev(w_scales, torch.uint8, "w_scales"), din, dout, None if bias is None else _b._dev(bias, torch.float32, "bias"),
        _b._dev(Y, Y.dtype, "Y"), _value(Y, "maxk_mx_linear: Y"), _b._stream()), "maxk_mx_linear")


def maxk_mx_matvec(X: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, Y: torch.Tensor, bias: Optional[torch.Tensor] = None) -> None:
    """Y [N, dout] is overwritten with X W^T + bias for few rows X [N, din] that are not rounded, W [dout, din] in 4 bits; X and Y each float32, bfloat16
    or float16.  16 rows cost up to twice what one does."""
    what = "maxk_mx_matvec"
    if _b._FAST is not None and _b._FAST.mx_matvec(X, w_codes, w_scales, Y, bias):
        return
    N, din = _matrix(X, f"{what}: X")
    if Y.dim() != 2 or Y.shape[0] != N:
        raise MaxKError(f"{what}: Y must be [N, dout]")
    dout = Y.shape[1]
    if dout > _MAX_CLASSES:
        _b._check(_UNSUPPORTED, what)
    _stored(w_codes, w_scales, dout, din, f"{what}: W", True)
    if bias is not None and tuple(bias.shape) != (dout,):
        raise MaxKError(f"{what}: bias must be [dout]")
    args = (_b._dev(X, X.dtype, "X"), _value(X, f"{what}: X"), N, _b._dev(w_codes, torch.uint8, "w_codes"), _b._dev(w_scales, torch.uint8, "w_scales"), din, dout,
            None if bias is None else _b._dev(bias, torch.float32, "bias"), _b._dev(Y, Y.dtype, "Y"), _value(Y, f"{what}: Y"))
    _b._here(what, X, w_codes, w_scales, Y, bias)
    _b._check(_b.load_library().maxk_mx_matvec(*args, _b._stream()), what)


def _weight_grad_shapes(codes, scales, N, dout, dW, db, what):
    rows, din = _matrix(dW, f"{what}: dW")
    fmt = _stored(codes, scales, N, din, what)
    if rows != dout or (db is not None and tuple(db.shape) != (dout,)):
        raise MaxKError(f"{what}: dW / db must be [dout, din] / [dout]")
    return din, fmt


def _workspace(workspace: Optional[torch.Tensor], N: int, din: int, dout: int, device, what: str) -> torch.Tensor:
    need = _b.load_library().maxk_mx_weight_grad_workspace(N, din, dout)
    if need < 0:
        _b._check(need, what)
    return torch.empty(need, dtype=torch.uint8, device=device) if workspace is None else workspace


def mx_weight_grad_workspace(N: int, din: int, dout: int) -> int:
    """Bytes that maxk_mx_weight_grad and maxk_mx_weight_grad_cbsr need as `workspace` (a uint8 tensor)."""
    what = "maxk_mx_weight_grad_workspace"
    need = int(_b.load_library().maxk_mx_weight_grad_workspace(N, _width(din, what), _width(dout, what)))
    if need < 0:
        _b._check(need, what)
    return need


def maxk_mx_weight_grad(codes: torch.Tensor, scales: torch.Tensor, dH: torch.Tensor, dW: torch.Tensor, db: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None) -> None:
    """dW [dout, din] and db [dout] (float32) are overwritten with dH^T X and the column sums of dH [N, dout] (float32, bfloat16,
    float16), X [N, din] stored in codes and scales.  workspace: uint8, from torch's allocator where none is given."""
    what = "maxk_mx_weight_grad"
    if _b._FAST is not None and _b._FAST.mx_weight_grad(codes, scales, dH, None, dW, db, workspace):
        return
    N, dout = _matrix(dH, f"{what}: dH")
    din, fmt = _weight_grad_shapes(codes, scales, N, dout, dW, db, what)
    args = (_b._dev(codes, codes.dtype, "codes"), _b._dev(scales, torch.uint8, "scales"), fmt, N, din, dout, _b._dev(dH, dH.dtype, "dH"),
            _value(dH, f"{what}: dH"), _b._dev(dW, torch.float32, "dW"), None if db is None else _b._dev(db, torch.float32, "db"))
    ws = _workspace(workspace, N, din, dout, dW.device, what)
    _b._check(_b.load_library().maxk_mx_weight_grad(*args, _b._dev(ws, torch.uint8, "workspace"), ws.numel(), _b._stream()), what)


def maxk_mx_weight_grad_cbsr(codes: torch.Tensor, scales: torch.Tensor, dXs: torch.Tensor, sp_index: torch.Tensor, dW: torch.Tensor,
                             db: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """maxk_mx_weight_grad for the gradient that maxk_sspmm_bwd leaves: dXs [N, k] float32 at the columns sp_index [N, k]."""
    what = "maxk_mx_weight_grad_cbsr"
    if _b._FAST is not None and _b._FAST.mx_weight_grad(codes, scales, dXs, sp_index, dW, db, workspace):
        return
    N, k = _matrix(dXs, f"{what}: dXs")
    dout = _width(_matrix(dW, f"{what}: dW")[0], f"{what}: dW")
    din, fmt = _weight_grad_shapes(codes, scales, N, dout, dW, db, what)
    ib = _index(sp_index, N, k, what)
    args = (_b._dev(codes, codes.dtype, "codes"), _b._dev(scales, torch.uint8, "scales"), fmt, N, din, dout, _b._dev(dXs, torch.float32, "dXs"),
            _b._dev(sp_index, sp_index.dtype, "sp_index"), ib, k, _b._dev(dW, torch.float32, "dW"),
            None if db is None else _b._dev(db, torch.float32, "db"))
    ws = _workspace(workspace, N, din, dout, dW.device, what)
    _b._check(_b.load_library().maxk_mx_weight_grad_cbsr(*args, _b._dev(ws, torch.uint8, "workspace"), ws.numel(), _b._stream()), what)


def _index(sp_index: torch.Tensor, N: int, k: int, what: str) -> int:
    if sp_index.dtype not in _b._INDEX_BYTES or tuple(sp_index.shape) != (N, k):
        raise MaxKError(f"{what}: sp_index must be [N, k] of uint8, uint16 or int32")
    return _b._INDEX_BYTES[sp_index.dtype]


def maxk_mx_input_grad(dH: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, dX: torch.Tensor) -> None:
    """dX [N, din] (float32, bfloat16, float16) is overwritten with dH W, dH [N, dout] in any of these types, W [dout, din] in 4 bits."""
    what = "maxk_mx_input_grad"
    if _b._FAST is not None and _b._FAST.mx_input_grad(dH, None, w_codes, w_scales, dX):
        return
    N, dout = _matrix(dH, f"{what}: dH")
    rows, din = _matrix(dX, f"{what}: dX")
    _stored(w_codes, w_scales, dout, din, f"{what}: W", True)
    if rows != N:
        raise MaxKError(f"{what}: dX must be [N, din]")
    _b._check(_b.load_library().maxk_mx_input_grad(
        _b._dev(dH, dH.dtype, "dH"), _value(dH, f"{what}: dH"), N, _b._dev(w_codes, torch.uint8, "w_codes"),
        _b._dev(w_scales, torch.uint8, "w_scales"), din, dout, _b._dev(dX, dX.dtype, "dX"), _value(dX, f"{what}: dX"), _b._stream()), what)


def maxk_mx_input_grad_cbsr(dXs: torch.Tensor, sp_index: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, dX: torch.Tensor) -> None:
    """maxk_mx_input_grad for the gradient that maxk_sspmm_bwd leaves."""
    what = "maxk_mx_input_grad_cbsr"
    if _b._FAST is not None and _b._FAST.mx_input_grad(dXs, sp_index, w_codes, w_scales, dX):
        return
    N, k = _matrix(dXs, f"{what}: dXs")
    rows, din = _matrix(dX, f"{what}: dX")
    dout = _width(_matrix(w_codes, f"{what}: W")[0], f"{what}: W")
    _stored(w_codes, w_scales, dout, din, f"{what}: W", True)
    ib = _index(sp_index, N, k, what)
    if rows != N:
        raise MaxKError(f"{what}: dX must be [N, din]")
    _b._check(_b.load_library().maxk_mx_input_grad_cbsr(
        _b._dev(dXs, torch.float32, "dXs"), _b._dev(sp_index, sp_index.dtype, "sp_index"), ib, k, N, _b._dev(w_codes, torch.uint8, "w_codes"),
        _b._dev(w_scales, torch.uint8, "w_scales"), din, dout, _b._dev(dX, dX.dtype, "dX"), _value(dX, f"{what}: dX"), _b._stream()), what)
