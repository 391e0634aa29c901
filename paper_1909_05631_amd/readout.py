"""The dense readout of a network's rows: softmax cross entropy with its gradient (ctypes binding of the calls in
include/sdnn.h that need no handle). Argument marshalling only: tensors are checked, nothing is computed or
allocated here. Every tensor lives on the GPU; rows may be strided, the values within a row may not.
`stream`: a torch stream, its handle, or None for the default stream."""
from __future__ import annotations

import torch

from .sdnn import _check, _stream_handle, load_library

DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _dtype(t: torch.dtype) -> int:
    if t not in DTYPES:
        raise ValueError(f"{t} is neither float32 nor bfloat16")
    return DTYPES[t]


def _on_gpu(name: str, t, like=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} is no tensor on the GPU")
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")


def _rows(name: str, t, shape, dtype, like=None) -> tuple[int, int]:
    """Address and row stride of a matrix of `shape` (None: any) and `dtype`."""
    _on_gpu(name, t, like)
    if t.dim() != 2 or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, not {dtype}")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"the values within a row of {name} are not contiguous")
    if rows > 1 and t.stride(0) < cols:
        raise ValueError(f"the rows of {name} overlap")
    return t.data_ptr(), t.stride(0) if rows > 1 else cols


def _vector(name: str, t, n: int, dtype, like) -> int:
    _on_gpu(name, t, like)
    if tuple(t.shape) != (n,) or t.dtype != dtype or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} is not {n} contiguous values of {dtype}")
    return t.data_ptr()


def _workspace(t, like) -> tuple[int | None, int]:
    _on_gpu("workspace", t, like)
    if not t.is_contiguous():
        raise ValueError("workspace is not contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def workspace_bytes(n_rows: int, n_classes: int, n_features: int, dtype: torch.dtype, gradient: bool = True) -> int:
    """Bytes of workspace for `loss`, or, with `gradient`, for `loss` and `gradient`."""
    return int(load_library().sdnn_readout_workspace_bytes(n_rows, n_classes, n_features, _dtype(dtype), int(gradient)))


def loss(x, w, labels, loss, lse, workspace, stream=None) -> None:
    """loss[t] = lse[t] - l[t, labels[t]] of the logits l = x w^T, lse[t] = log sum_v exp l[t, v]; 0 where the label
    is outside the classes. x (rows, features), w (classes, features): float32 or bfloat16. labels: int64. loss,
    lse (or None): float32, written."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, (None, None), x.dtype)
    pw, ldw = _rows("w", w, (None, x.shape[1]), x.dtype, x)
    n, ws = x.shape[0], _workspace(workspace, x)
    with torch.cuda.device(x.device):
        _check(load_library().sdnn_readout_loss(
            px, ldx, pw, ldw, dt, _vector("labels", labels, n, torch.int64, x), n, w.shape[0], x.shape[1],
            _vector("loss", loss, n, torch.float32, x), None if lse is None else _vector("lse", lse, n, torch.float32, x),
            *ws, _stream_handle(stream)))


def gradient(x, w, labels, lse, dx, dw, workspace, row_grad=None, stream=None) -> None:
    """The gradients of sum_t row_grad[t] loss[t] (None: of the mean loss over the rows with a label) to x and w,
    written to dx and dw (either may be None) in their type; lse as `loss` left it."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, (None, None), x.dtype)
    pw, ldw = _rows("w", w, (None, x.shape[1]), x.dtype, x)
    pdx, lddx = (None, 0) if dx is None else _rows("dx", dx, x.shape, x.dtype, x)
    pdw, lddw = (None, 0) if dw is None else _rows("dw", dw, w.shape, x.dtype, x)
    n, ws = x.shape[0], _workspace(workspace, x)
    with torch.cuda.device(x.device):
        _check(load_library().sdnn_readout_grad(
            px, ldx, pw, ldw, dt, _vector("labels", labels, n, torch.int64, x), _vector("lse", lse, n, torch.float32, x),
            None if row_grad is None else _vector("row_grad", row_grad, n, torch.float32, x), n, w.shape[0], x.shape[1],
            pdx, lddx, pdw, lddw, *ws, _stream_handle(stream)))
