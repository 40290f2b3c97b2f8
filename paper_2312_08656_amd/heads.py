"""Both ends of a classifier: the norm in front of a layer, log probabilities of classes and distillation behind the last one (see include/maxk.h for the
contract of each call).

Matrices are float32, bfloat16 or float16, vectors float32.  As in the rest of the binding, outputs are given by the caller and overwritten, tensors are
contiguous, and every call enqueues on the current stream; tensors are those of the current device.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as _b
from .binding import MaxKError
from .mx import _MAX_CLASSES, _UNSUPPORTED, _stored, _value

_NORM_MAX_DIM = 16384  # MAXK_NORM_MAX_DIM
_LABEL_BYTES = {torch.int32: 4, torch.int64: 8}


def _rows(t: torch.Tensor, most: int, what: str):
    """(N, width) of a matrix whose width the call takes."""
    if t.dim() != 2:
        raise MaxKError(f"{what}: expected a matrix")
    if t.shape[1] > most:
        _b._check(_UNSUPPORTED, what)
    return t.shape[0], t.shape[1]


def _like(t: Optional[torch.Tensor], X: torch.Tensor, what: str) -> Optional[int]:
    """Address of a matrix of X's shape and type, None where there is none."""
    if t is None:
        return None
    if t.shape != X.shape:
        raise MaxKError(f"{what}: expected a matrix of shape {tuple(X.shape)}")
    return _b._dev(t, X.dtype, what)


def _vector(t: Optional[torch.Tensor], n: int, what: str) -> Optional[int]:
    if t is None:
        return None
    if tuple(t.shape) != (n,):
        raise MaxKError(f"{what}: expected [{n}]")
    return _b._dev(t, torch.float32, what)


def _room(workspace: Optional[torch.Tensor], need: int, device, what: str):
    """(address, bytes) of the workspace, from torch's allocator where none is given."""
    if need < 0:
        _b._check(need, what)
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return _b._dev(workspace, torch.uint8, f"{what}: workspace"), workspace.numel(), workspace


def maxk_rms_norm(X: torch.Tensor, gamma: torch.Tensor, Y: Optional[torch.Tensor] = None, codes: Optional[torch.Tensor] = None,
                  scales: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, H: Optional[torch.Tensor] = None,
                  rstd: Optional[torch.Tensor] = None, eps: float = 1e-6) -> None:
    """H = X + residual; Y = H r gamma with r = 1 / sqrt(mean of a row's H^2 + eps), X [N, dim], gamma [dim] float32.

    Y is overwritten in X's type (Y), in 8 or 4 bits (codes and scales, see mx_empty), or both, rstd [N] with r.  eps is 8.64e-78 at least.  residual and H are given together, and H may be either
    operand itself; without them H is X."""
    what = "maxk_rms_norm"
    if _b._FAST is not None and _b._FAST.rms_norm(X, gamma, Y, codes, scales, residual, H, rstd, eps):
        return
    N, dim = _rows(X, _NORM_MAX_DIM, f"{what}: X")
    if (residual is None) != (H is None) or (codes is None) != (scales is None) or (Y is None and codes is None):
        raise MaxKError(f"{what}: residual and H, and codes and scales, go together, and Y or codes must be given")
    fmt = 0 if codes is None else _stored(codes, scales, N, dim, what)
    args = (_b._dev(X, X.dtype, "X"), _like(residual, X, f"{what}: residual"), _value(X, f"{what}: X"), N, dim, _vector(gamma, dim, f"{what}: gamma"), eps,
            _like(H, X, f"{what}: H"), _like(Y, X, f"{what}: Y"), fmt, None if codes is None else _b._dev(codes, codes.dtype, "codes"),
            None if scales is None else _b._dev(scales, torch.uint8, "scales"), _vector(rstd, N, f"{what}: rstd"))
    _b._here(what, X, gamma, Y, codes, scales, residual, H, rstd)
    _b._check(_b.load_library().maxk_rms_norm(*args, _b._stream()), what)


def rms_norm_grad_workspace(N: int, dim: int) -> int:
    """Bytes that maxk_rms_norm_grad needs as `workspace` (a uint8 tensor) where it computes dgamma."""
    what = "maxk_rms_norm_grad_workspace"
    if dim > _NORM_MAX_DIM:
        _b._check(_UNSUPPORTED, what)
    need = int(_b.load_library().maxk_rms_norm_grad_workspace(N, dim))
    if need < 0:
        _b._check(need, what)
    return need


def maxk_rms_norm_grad(dY: torch.Tensor, H: torch.Tensor, gamma: torch.Tensor, rstd: torch.Tensor, dX: torch.Tensor, dgamma: Optional[torch.Tensor] = None,
                       dH: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """dX [N, dim] (of X and of the residual alike) and dgamma [dim] are overwritten with the gradients of maxk_rms_norm, for the H and rstd that it left.

    dH: the gradient that arrives at H beside dY.  dX may be dY or dH itself.  workspace: uint8, from torch's allocator where none is given."""
    what = "maxk_rms_norm_grad"
    if _b._FAST is not None and _b._FAST.rms_norm_grad(dY, H, gamma, rstd, dX, dgamma, dH, workspace):
        return
    N, dim = _rows(H, _NORM_MAX_DIM, f"{what}: H")
    args = (_like(dY, H, f"{what}: dY"), _b._dev(H, H.dtype, "H"), _like(dH, H, f"{what}: dH"), _value(H, f"{what}: H"), N, dim,
            _vector(gamma, dim, f"{what}: gamma"), _vector(rstd, N, f"{what}: rstd"), _like(dX, H, f"{what}: dX"), _vector(dgamma, dim, f"{what}: dgamma"))
    _b._here(what, dY, H, gamma, rstd, dX, dgamma, dH, workspace)
    at, size, _held = _room(workspace, rms_norm_grad_workspace(N, dim) if dgamma is not None else 0, H.device, what)
    _b._check(_b.load_library().maxk_rms_norm_grad(*args, at, size, _b._stream()), what)


def classes_workspace(N: int, V: int, k: int = 0) -> int:
    """Bytes (0: none) that the calls on logits [N, V] need as `workspace` (a uint8 tensor); k: alternatives of maxk_logprobs, else 0."""
    what = "maxk_classes_workspace"
    if V > _MAX_CLASSES:
        _b._check(_UNSUPPORTED, what)
    need = int(_b.load_library().maxk_classes_workspace(N, V, min(k, 1 << 30)))
    if need < 0:
        _b._check(need, what)
    return need


def _labels(labels: Optional[torch.Tensor], N: int, what: str):
    if labels is None:
        return None, 0
    if labels.dtype not in _LABEL_BYTES or tuple(labels.shape) != (N,):
        raise MaxKError(f"{what}: labels must be [N] of int32 or int64")
    return _b._dev(labels, labels.dtype, f"{what}: labels"), _LABEL_BYTES[labels.dtype]


def maxk_logprobs(logits: torch.Tensor, labels: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                  top_data: Optional[torch.Tensor] = None, top_index: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """Of each row of logits [N, V]: logprob [N] of its class in labels [N] (int32 or int64; negative: none, 0), entropy [N], and the k likeliest classes,
    likeliest first: top_data [N, k] (float32) their log probabilities, top_index [N, k] (uint8, uint16 or int32) their columns.  Those that are given are
    overwritten."""
    what = "maxk_logprobs"
    if _b._FAST is not None and _b._FAST.logprobs(logits, labels, logprob, entropy, top_data, top_index, workspace):
        return
    N, V = _rows(logits, _MAX_CLASSES, f"{what}: logits")
    if (top_data is None) != (top_index is None) or (logprob is not None and labels is None) or (logprob is None and entropy is None and top_data is None):
        raise MaxKError(f"{what}: top_data and top_index go together, logprob needs labels, and something must be asked for")
    k = ib = 0
    if top_data is not None:
        if top_data.dim() != 2 or top_data.shape[0] != N or top_index.shape != top_data.shape or top_index.dtype not in _b._INDEX_BYTES:
            raise MaxKError(f"{what}: top_data / top_index must be [N, k], top_index of uint8, uint16 or int32")
        k, ib = top_data.shape[1], _b._INDEX_BYTES[top_index.dtype]
        if k < 1:
            raise MaxKError(f"{what}: k must be at least 1")
    at, label_bytes = _labels(labels, N, what)
    args = (_b._dev(logits, logits.dtype, "logits"), _value(logits, f"{what}: logits"), N, V, at, label_bytes, _vector(logprob, N, f"{what}: logprob"),
            _vector(entropy, N, f"{what}: entropy"), None if top_data is None else _b._dev(top_data, torch.float32, "top_data"),
            None if top_index is None else _b._dev(top_index, top_index.dtype, "top_index"), ib, k)
    _b._here(what, logits, labels, logprob, entropy, top_data, top_index, workspace)
    room, size, _held = _room(workspace, classes_workspace(N, V, k), logits.device, what)
    _b._check(_b.load_library().maxk_logprobs(*args, room, size, _b._stream()), what)


def maxk_logprobs_grad(logits: torch.Tensor, dlogits: torch.Tensor, labels: Optional[torch.Tensor] = None, dlogprob: Optional[torch.Tensor] = None,
                       dentropy: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None) -> None:
    """dlogits [N, V] (in the logits' type, and may be the logits themselves) is overwritten with the gradient of sum(dlogprob * logprob + dentropy * entropy), either [N] or
    None.  logprob and entropy, where given, with those of maxk_logprobs: a training step whose weights are known is this one call."""
    what = "maxk_logprobs_grad"
    if _b._FAST is not None and _b._FAST.logprobs_grad(logits, dlogits, labels, dlogprob, dentropy, logprob, entropy, workspace):
        return
    N, V = _rows(logits, _MAX_CLASSES, f"{what}: logits")
    if (dlogprob is None and dentropy is None) or (labels is None and (dlogprob is not None or logprob is not None)):
        raise MaxKError(f"{what}: dlogprob or dentropy must be given, and dlogprob and logprob need labels")
    at, label_bytes = _labels(labels, N, what)
    args = (_b._dev(logits, logits.dtype, "logits"), _value(logits, f"{what}: logits"), N, V, at, label_bytes, _vector(dlogprob, N, f"{what}: dlogprob"),
            _vector(dentropy, N, f"{what}: dentropy"), _vector(logprob, N, f"{what}: logprob"), _vector(entropy, N, f"{what}: entropy"),
            _like(dlogits, logits, f"{what}: dlogits"))
    _b._here(what, logits, dlogits, labels, dlogprob, dentropy, logprob, entropy, workspace)
    room, size, _held = _room(workspace, classes_workspace(N, V), logits.device, what)
    _b._check(_b.load_library().maxk_logprobs_grad(*args, room, size, _b._stream()), what)


def _teacher(top_data: torch.Tensor, top_index: torch.Tensor, N: int, what: str):
    if top_data.dim() != 2 or top_data.shape[0] != N or top_index.shape != top_data.shape or top_index.dtype not in _b._INDEX_BYTES:
        raise MaxKError(f"{what}: top_data / top_index must be [N, k], top_index of uint8, uint16 or int32")
    return (_b._dev(top_data, top_data.dtype, "top_data"), _value(top_data, f"{what}: top_data"), _b._dev(top_index, top_index.dtype, "top_index"),
            _b._INDEX_BYTES[top_index.dtype], min(top_data.shape[1], 1 << 30))


def maxk_distill(logits: torch.Tensor, top_data: torch.Tensor, top_index: torch.Tensor, loss: torch.Tensor, temperature: float = 1.0,
                 workspace: Optional[torch.Tensor] = None) -> None:
    """loss [N] is overwritten with the divergence of softmax(logits / temperature), logits [N, V], from the softmax of the k logits a row that a teacher passed on:
    top_data [N, k] (any of the types) / temperature at the columns top_index [N, k] (uint8, uint16 or int32), k up to V and 1024.  Entries of -inf or outside [0, V) are
    none.  temperature: from 4.24e-39 to fp32's largest value."""
    what = "maxk_distill"
    if _b._FAST is not None and _b._FAST.distill(logits, top_data, top_index, None, None, temperature, loss, workspace):
        return
    N, V = _rows(logits, _MAX_CLASSES, f"{what}: logits")
    teacher = _teacher(top_data, top_index, N, what)
    args = (_b._dev(logits, logits.dtype, "logits"), _value(logits, f"{what}: logits"), N, V, *teacher, temperature,
            _vector(loss, N, f"{what}: loss"))
    _b._here(what, logits, top_data, top_index, loss, workspace)
    room, size, _held = _room(workspace, classes_workspace(N, V), logits.device, what)
    _b._check(_b.load_library().maxk_distill(*args, room, size, _b._stream()), what)


def maxk_distill_grad(logits: torch.Tensor, top_data: torch.Tensor, top_index: torch.Tensor, dloss: torch.Tensor, dlogits: torch.Tensor,
                      temperature: float = 1.0, loss: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> None:
    """dlogits [N, V] (in the logits' type, and may be the logits themselves) is overwritten with the gradient of sum(dloss * loss), dloss [N].  loss, where
    given, with that of maxk_distill: a training step whose weights are known is this one call."""
    what = "maxk_distill_grad"
    if _b._FAST is not None and _b._FAST.distill(logits, top_data, top_index, dloss, dlogits, temperature, loss, workspace):
        return
    N, V = _rows(logits, _MAX_CLASSES, f"{what}: logits")
    teacher = _teacher(top_data, top_index, N, what)
    args = (_b._dev(logits, logits.dtype, "logits"), _value(logits, f"{what}: logits"), N, V, *teacher, temperature,
            _vector(dloss, N, f"{what}: dloss"), _vector(loss, N, f"{what}: loss"), _like(dlogits, logits, f"{what}: dlogits"))
    _b._here(what, logits, top_data, top_index, dloss, dlogits, loss, workspace)
    room, size, _held = _room(workspace, classes_workspace(N, V), logits.device, what)
    _b._check(_b.load_library().maxk_distill_grad(*args, room, size, _b._stream()), what)
