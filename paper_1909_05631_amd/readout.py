"""The dense readout of a network's rows: softmax cross entropy with its gradient, orthogonalised updates, and products
of microscaled 4-bit floats (ctypes binding of the calls in include/sdnn.h that need no handle). Argument marshalling only: tensors are checked, nothing is computed or
allocated here. Every tensor lives on the GPU; rows may be strided, the values within a row may not.
`stream`: a torch stream, its handle, or None for the default stream."""
from __future__ import annotations

import ctypes

import torch

from .sdnn import SdnnError, _check, _stream_handle, load_library  # noqa: F401

DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _dtype(t: torch.dtype) -> int:
    code = DTYPES.get(t)
    if code is None:
        raise ValueError(f"{t} is neither float32 nor bfloat16")
    return code


def _on_gpu(name: str, t, like=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} is no tensor on the GPU")
    if like is not None and t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")


def _rows(name: str, t, rows, cols, dtype, like=None) -> tuple[int, int]:
    """Address and row stride of a matrix of rows x cols (None: any) and `dtype`."""
    _on_gpu(name, t, like)
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ValueError(f"{name} has shape {tuple(shape)}, not ({rows}, {cols})")
    if t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, not {dtype}")
    m, n = shape
    ld, step = t.stride()
    if n > 1 and step != 1:
        raise ValueError(f"the values within a row of {name} are not contiguous")
    if m > 1 and ld < n:
        raise ValueError(f"the rows of {name} overlap")
    return t.data_ptr(), ld if m > 1 else n


def _vector(name: str, t, n: int, dtype, like) -> int:
    _on_gpu(name, t, like)
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} is not {n} contiguous values of {dtype}")
    return t.data_ptr()


def _workspace(t, like) -> tuple[int | None, int]:
    _on_gpu("workspace", t, like)
    if not t.is_contiguous():
        raise ValueError("workspace is not contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def _call(like, name: str, *args) -> None:
    """The library's call, on the device of `like`."""
    entry = getattr(load_library(), name)
    if torch.cuda.current_device() == like.get_device():
        status = entry(*args)
    else:
        with torch.cuda.device(like.device):
            status = entry(*args)
    if status:
        _check(status)


def workspace_bytes(n_rows: int, n_classes: int, n_features: int, dtype: torch.dtype, gradient: bool = True) -> int:
    """Bytes of workspace for `loss`, or, with `gradient`, for `loss` and `gradient`."""
    return int(load_library().sdnn_readout_workspace_bytes(n_rows, n_classes, n_features, _dtype(dtype), int(gradient)))


def loss(x, w, labels, loss, lse, workspace, stream=None) -> None:
    """loss[t] = lse[t] - l[t, labels[t]] of the logits l = x w^T, lse[t] = log sum_v exp l[t, v]; 0 where the label
    is outside the classes. x (rows, features), w (classes, features): float32 or bfloat16. labels: int64. loss,
    lse (or None): float32, written."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, None, None, x.dtype)
    n, d = x.shape
    pw, ldw = _rows("w", w, None, d, x.dtype, x)
    _call(x, "sdnn_readout_loss", px, ldx, pw, ldw, dt, _vector("labels", labels, n, torch.int64, x), n, w.shape[0], d,
          _vector("loss", loss, n, torch.float32, x), None if lse is None else _vector("lse", lse, n, torch.float32, x),
          *_workspace(workspace, x), _stream_handle(stream))


def gradient(x, w, labels, lse, dx, dw, workspace, row_grad=None, stream=None) -> None:
    """The gradients of sum_t row_grad[t] loss[t] (None: of the mean loss over the rows with a label) to x and w,
    written to dx and dw (either may be None) in their type; lse as `loss` left it."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, None, None, x.dtype)
    n, d = x.shape
    pw, ldw = _rows("w", w, None, d, x.dtype, x)
    v = w.shape[0]
    pdx, lddx = (None, 0) if dx is None else _rows("dx", dx, n, d, x.dtype, x)
    pdw, lddw = (None, 0) if dw is None else _rows("dw", dw, v, d, x.dtype, x)
    _call(x, "sdnn_readout_grad", px, ldx, pw, ldw, dt, _vector("labels", labels, n, torch.int64, x),
          _vector("lse", lse, n, torch.float32, x), None if row_grad is None else _vector("row_grad", row_grad, n, torch.float32, x),
          n, v, d, pdx, lddx, pdw, lddw, *_workspace(workspace, x), _stream_handle(stream))


def orthogonalize_workspace_bytes(batch: int, rows: int, cols: int) -> int:
    return int(load_library().sdnn_orthogonalize_workspace_bytes(batch, rows, cols))


def _matrices(name: str, t, like=None) -> tuple[int, int, int]:
    """Address, row stride and batch stride of one matrix or a batch of them."""
    _on_gpu(name, t, like)
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} is neither a matrix nor a batch of them")
    if 0 in t.shape[-2:]:
        raise ValueError(f"the matrices of {name} are empty")
    if t.numel() == 0:  # a batch of none
        return t.data_ptr(), t.shape[2], 0
    p, ld = _rows(name, t if t.dim() == 2 else t[0], None, None, t.dtype)
    return p, ld, t.stride(0) if t.dim() == 3 else 0


def orthogonalize(g, out, workspace, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  stream=None) -> None:
    """out = g (a matrix, or a batch of them) orthogonalised by `steps` Newton-Schulz products; out may be g itself."""
    try:
        a, b, c = (float(v) for v in coefficients)
    except (TypeError, ValueError) as e:
        raise ValueError(f"coefficients {coefficients!r} are not three numbers") from e
    _on_gpu("g", g)
    dt = _dtype(g.dtype)
    pg, ldg, batch_g = _matrices("g", g)
    _on_gpu("out", out, g)
    if tuple(out.shape) != tuple(g.shape) or out.dtype != g.dtype:
        raise ValueError(f"out is {tuple(out.shape)} of {out.dtype}, not {tuple(g.shape)} of {g.dtype}")
    po, ldo, batch_o = _matrices("out", out, g)
    batch, (rows, cols) = g.shape[0] if g.dim() == 3 else 1, g.shape[-2:]
    coef = (ctypes.c_float * 3)(a, b, c)
    _call(g, "sdnn_orthogonalize", pg, ldg, batch_g, po, ldo, batch_o, dt, batch, rows, cols, steps, coef, eps,
          *_workspace(workspace, g), _stream_handle(stream))


def mx_blocks(n_values: int) -> int:
    """Blocks of 32 values that hold a row of n_values: 16 bytes of codes and one of scale each (sdnn_mx_blocks)."""
    return 4 * -(-n_values // 128) if 1 <= n_values <= 1 << 20 else 0


def mx_linear_workspace_bytes(n_rows: int, n_values: int) -> int:
    return int(load_library().sdnn_mx_linear_workspace_bytes(n_rows, n_values))


def _codes(name: str, codes, scales, n_values: int, like) -> tuple[int, int, int]:
    """Addresses of codes and scales, and their rows."""
    _on_gpu(f"the codes of {name}", codes, like)
    _on_gpu(f"the scales of {name}", scales, like)
    n, rows = mx_blocks(n_values), codes.shape[0] if codes.dim() else 0
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError(f"the codes and scales of {name} are not contiguous bytes")
    if tuple(codes.shape) != (rows, 16 * n) or tuple(scales.shape) != (rows, n):
        raise ValueError(f"codes {tuple(codes.shape)} and scales {tuple(scales.shape)} of {name} do not hold rows of {n_values} values")
    return codes.data_ptr(), scales.data_ptr(), rows


def mx_quantize(x, codes, scales, stream=None) -> None:
    """codes (rows, 16 * mx_blocks(n)) and scales (rows, mx_blocks(n)), bytes, of x (rows, n)."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, None, None, x.dtype)
    pc, ps, rows = _codes("x", codes, scales, x.shape[1], x)
    if rows != x.shape[0]:
        raise ValueError(f"{rows} rows of codes for {x.shape[0]} rows of x")
    _call(x, "sdnn_mx_quantize", px, ldx, dt, rows, x.shape[1], pc, ps, _stream_handle(stream))


def mx_dequantize(codes, scales, out, stream=None) -> None:
    """out (rows, n) = the values that the codes stand for."""
    _on_gpu("out", out)
    dt = _dtype(out.dtype)
    po, ldo = _rows("out", out, None, None, out.dtype)
    pc, ps, rows = _codes("the input", codes, scales, out.shape[1], out)
    if rows != out.shape[0]:
        raise ValueError(f"{rows} rows of codes for {out.shape[0]} rows of out")
    _call(out, "sdnn_mx_dequantize", pc, ps, rows, out.shape[1], po, ldo, dt, _stream_handle(stream))


def mx_product(x_codes, x_scales, w_codes, w_scales, n_values: int, out, stream=None) -> None:
    """out (rows, outputs) = x w^T of quantised rows of n_values values."""
    _on_gpu("out", out)
    dt = _dtype(out.dtype)
    pxc, pxs, rows = _codes("x", x_codes, x_scales, n_values, out)
    pwc, pws, outputs = _codes("w", w_codes, w_scales, n_values, out)
    po, ldo = _rows("out", out, rows, outputs, out.dtype)
    _call(out, "sdnn_mx_product", pxc, pxs, pwc, pws, rows, outputs, n_values, po, ldo, dt, _stream_handle(stream))


def mx_linear(x, w_codes, w_scales, out, workspace, stream=None) -> None:
    """out (rows, outputs) = x w^T, x (rows, n) quantised on the way; out has x's type."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, None, None, x.dtype)
    pwc, pws, outputs = _codes("w", w_codes, w_scales, x.shape[1], x)
    po, ldo = _rows("out", out, x.shape[0], outputs, x.dtype, x)
    _call(x, "sdnn_mx_linear", px, ldx, dt, pwc, pws, x.shape[0], outputs, x.shape[1], po, ldo, *_workspace(workspace, x),
          _stream_handle(stream))
