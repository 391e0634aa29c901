"""The dense readout of a network's rows: softmax cross entropy with its gradient, orthogonalised updates, products
of microscaled 4-bit floats, a gated hidden layer under it, gradients clipped by their norm, and weights of 4 bits with a
scale a group (ctypes binding of the calls in include/sdnn.h that need no handle). Argument marshalling only: tensors are checked, nothing is computed or
allocated here. Every tensor lives on the GPU; rows may be strided, the values within a row may not.
`stream`: a torch stream, its handle, or None for the default stream."""
from __future__ import annotations

import ctypes
from operator import attrgetter

import numpy as np
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


ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}


def _activation(name) -> int:
    code = ACTIVATIONS.get(name) if isinstance(name, str) else None
    if code is None:
        raise ValueError(f"activation {name!r} is none of {', '.join(ACTIVATIONS)}")
    return code


def gated_workspace_bytes(n_rows: int, n_hidden: int, n_features: int, dtype: torch.dtype, gradient: bool = True, kept: bool = True) -> int:
    """Bytes of workspace for `gated`, or, with `gradient`, for `gated` and `gated_gradient`; kept=False: also where that
    gets no gate and up."""
    return int(load_library().sdnn_gated_workspace_bytes(n_rows, n_hidden, n_features, _dtype(dtype), (1 if kept else 2) if gradient else 0))


def _layer(x, w_gate, w_up):
    """dtype, (rows, hidden, features) and the leading arguments of a gated layer's calls."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, None, None, x.dtype)
    n, d = x.shape
    pg, ldg = _rows("w_gate", w_gate, None, d, x.dtype, x)
    pu, ldu = _rows("w_up", w_up, w_gate.shape[0], d, x.dtype, x)
    return (n, w_gate.shape[0], d), (px, ldx, pg, ldg, pu, ldu, dt)


def _optional_rows(name: str, t, rows, cols, dtype, like) -> tuple[int | None, int]:
    return (None, 0) if t is None else _rows(name, t, rows, cols, dtype, like)


def gated(x, w_gate, w_up, h, workspace, activation: str = "silu", gate=None, up=None, stream=None) -> None:
    """h (rows, hidden) = act(x w_gate^T) * (x w_up^T): x (rows, features), w_gate, w_up (hidden, features), float32 or
    bfloat16; activation "silu", "gelu" or "relu". gate, up (or None): like h, the two products, for `gated_gradient`."""
    act = _activation(activation)
    (n, m, d), lead = _layer(x, w_gate, w_up)
    _call(x, "sdnn_gated", *lead, act, n, m, d, *_rows("h", h, n, m, x.dtype, x), *_optional_rows("gate", gate, n, m, x.dtype, x),
          *_optional_rows("up", up, n, m, x.dtype, x), *_workspace(workspace, x), _stream_handle(stream))


def gated_gradient(x, w_gate, w_up, dh, dx, dw_gate, dw_up, workspace, activation: str = "silu", gate=None, up=None, stream=None) -> None:
    """From the gradient dh of h: dx, dw_gate and dw_up (each may be None), written in x's type; gate and up as `gated`
    kept them (None: computed again)."""
    act = _activation(activation)
    (n, m, d), lead = _layer(x, w_gate, w_up)
    _call(x, "sdnn_gated_grad", *lead, act, *_optional_rows("gate", gate, n, m, x.dtype, x), *_optional_rows("up", up, n, m, x.dtype, x),
          *_rows("dh", dh, n, m, x.dtype, x), n, m, d, *_optional_rows("dx", dx, n, d, x.dtype, x),
          *_optional_rows("dw_gate", dw_gate, m, d, x.dtype, x), *_optional_rows("dw_up", dw_up, m, d, x.dtype, x),
          *_workspace(workspace, x), _stream_handle(stream))


def clip_workspace_bytes(n_tensors: int) -> int:
    """Bytes of workspace for `global_norm` and `clip` of so many tensors, whatever their sizes."""
    return int(load_library().sdnn_clip_workspace_bytes(n_tensors))


def _extent(name: str, t) -> tuple[int, int, int]:
    """Rows, columns and row stride of a tensor that is contiguous or a matrix of contiguous rows."""
    if t.is_contiguous():
        return 1, t.numel(), 0
    if t.dim() != 2:
        raise ValueError(f"{name} is neither contiguous nor a matrix of contiguous rows")
    return *t.shape, _rows(name, t, None, None, t.dtype)[1]


def _asked(name: str, tensors, norm) -> tuple[list, list]:
    """Types and addresses of a list of tensors on the GPU of `norm`. A list may hold hundreds: what is asked of all of
    them is asked by map, which costs a tenth of a microsecond a tensor."""
    for kind in set(map(type, tensors)):
        if not issubclass(kind, torch.Tensor):
            raise ValueError(f"{name} holds a {kind.__name__}, which is no tensor")
    if set(map(torch.Tensor.get_device, tensors)) - {norm.get_device()}:
        raise ValueError(f"not all of {name} are on the GPU of norm, {norm.device}")
    return list(map(attrgetter("dtype"), tensors)), list(map(torch.Tensor.data_ptr, tensors))


def _refuse_pair(tensors, to) -> None:
    """Refuses an output of another type than its tensor's, or of other values: of another number where both are contiguous, of
    another shape otherwise."""
    for i, (a, b) in enumerate(zip(tensors, to)):
        flat = a.is_contiguous() and b.is_contiguous()
        if a.dtype != b.dtype or (a.numel() != b.numel() if flat else a.shape != b.shape):
            raise ValueError(f"out[{i}] is {tuple(b.shape)} of {b.dtype}, not {tuple(a.shape)} of {a.dtype}")


def _list(tensors, out, norm):
    """The C ABI's description of a list of tensors (sdnn_tensor, seven words each) and its length."""
    _on_gpu("norm", norm)
    tensors = list(tensors)
    to = tensors if out is None else list(out)
    n = len(tensors)
    if len(to) != n:
        raise ValueError(f"out holds {len(to)} tensors, not {n}")
    dtypes, addresses = _asked("tensors", tensors, norm)
    to_dtypes, to_addresses = (dtypes, addresses) if to is tensors else _asked("out", to, norm)
    codes = list(map(DTYPES.get, dtypes))
    if None in codes:
        _dtype(dtypes[codes.index(None)])
    table = np.zeros((n, 7), np.int64)
    table[:, 0], table[:, 6] = addresses, codes
    table[:, 1] = table[:, 0] if to is tensors else to_addresses
    flat = all(map(torch.Tensor.is_contiguous, tensors)) and (to is tensors or all(map(torch.Tensor.is_contiguous, to)))
    if flat:
        shapes = list(map(torch.Tensor.numel, tensors))
        if to is not tensors and (dtypes != to_dtypes or shapes != list(map(torch.Tensor.numel, to))):
            _refuse_pair(tensors, to)
        table[:, 2], table[:, 3] = 1, shapes
    else:
        if to is not tensors:
            _refuse_pair(tensors, to)
        for i, (a, b) in enumerate(zip(tensors, to)):
            (rows, cols, ld), (rows_out, cols_out, ldo) = _extent(f"tensors[{i}]", a), _extent(f"out[{i}]", b)
            if rows != rows_out or cols != cols_out:  # one of them is contiguous, the other a matrix of rows
                rows, cols = a.shape
                ld, ldo = ld or cols, ldo or cols
            table[i, 2:6] = rows, cols, ld, ldo
    return table, n


def global_norm(tensors, norm, workspace, stream=None) -> None:
    """norm (1 value, float32) = the square root of the sum of squares of all values of the tensors, float32 or
    bfloat16, each contiguous or a matrix of contiguous rows."""
    table, n = _list(tensors, None, norm)
    _call(norm, "sdnn_global_norm", table.ctypes.data, n, _vector("norm", norm, 1, torch.float32, norm), *_workspace(workspace, norm),
          _stream_handle(stream))


def clip(tensors, max_norm: float, norm, workspace, out=None, stream=None) -> None:
    """The norm, as `global_norm` has it, and every value times min(1, max_norm / norm), into the tensors of `out` (of the same
    types and shapes; next to a contiguous tensor, a contiguous one of as many values; None: the tensors themselves)."""
    table, n = _list(tensors, out, norm)
    _call(norm, "sdnn_clip", table.ctypes.data, n, max_norm, _vector("norm", norm, 1, torch.float32, norm), *_workspace(workspace, norm),
          _stream_handle(stream))


GROUPS = (32, 64, 128)


def grouped_groups(n_values: int, group: int = 128) -> int:
    """Groups of a row of n_values weights: group / 2 bytes of codes and one scale each (sdnn_grouped_groups)."""
    return -(-n_values // group) if 1 <= n_values <= 1 << 20 and group in GROUPS else 0


def _whole(name: str, t, rows: int, cols: int, dtype, like) -> int:
    """Address of a contiguous matrix."""
    _on_gpu(name, t, like)
    if t.dtype != dtype or t.shape != (rows, cols) or not t.is_contiguous():
        raise ValueError(f"{name}, {tuple(t.shape)} of {t.dtype}, is not ({rows}, {cols}) contiguous values of {dtype}")
    return t.data_ptr()


def _grouped(codes, scales, offsets, n_values: int, group: int, dtype, like) -> tuple[int, int, int | None, int]:
    """Addresses of codes, scales and offsets, and their rows."""
    if not isinstance(group, int) or group not in GROUPS:
        raise ValueError(f"group {group!r} is none of {', '.join(map(str, GROUPS))}")
    n = grouped_groups(n_values, group)
    _on_gpu("codes", codes, like)
    rows = codes.shape[0] if codes.dim() else 0
    return (_whole("codes", codes, rows, n * group // 2, torch.uint8, like), _whole("scales", scales, rows, n, dtype, like),
            None if offsets is None else _whole("offsets", offsets, rows, n, dtype, like), rows)


def grouped_quantize(w, codes, scales, group: int = 128, offsets=None, stream=None) -> None:
    """codes (rows, group / 2 * n), bytes, and scales (rows, n), in w's type, of w (rows, values), n = grouped_groups(values,
    group): w = scale * (code - 8), or with offsets (rows, n) scale * code + offset."""
    _on_gpu("w", w)
    dt = _dtype(w.dtype)
    pw, ldw = _rows("w", w, None, None, w.dtype)
    pc, ps, po, rows = _grouped(codes, scales, offsets, w.shape[1], group, w.dtype, w)
    if rows != w.shape[0]:
        raise ValueError(f"{rows} rows of codes for {w.shape[0]} rows of w")
    _call(w, "sdnn_grouped_quantize", pw, ldw, dt, rows, w.shape[1], group, pc, ps, po, _stream_handle(stream))


def grouped_dequantize(codes, scales, out, group: int = 128, offsets=None, stream=None) -> None:
    """out (rows, values) = the weights that the codes stand for, in the scales' type."""
    _on_gpu("out", out)
    dt = _dtype(out.dtype)
    po, ldo = _rows("out", out, None, None, out.dtype)
    pc, ps, pf, rows = _grouped(codes, scales, offsets, out.shape[1], group, out.dtype, out)
    if rows != out.shape[0]:
        raise ValueError(f"{rows} rows of codes for {out.shape[0]} rows of out")
    _call(out, "sdnn_grouped_dequantize", pc, ps, pf, dt, rows, out.shape[1], group, po, ldo, _stream_handle(stream))


def grouped_linear_workspace_bytes(n_rows: int, n_outputs: int, n_values: int, dtype: torch.dtype) -> int:
    return int(load_library().sdnn_grouped_linear_workspace_bytes(n_rows, n_outputs, n_values, _dtype(dtype)))


def grouped_linear(x, codes, scales, out, workspace, group: int = 128, offsets=None, stream=None) -> None:
    """out (rows, outputs) = x w^T, x (rows, values), of weights held in 4 bits; scales, offsets and out have x's type."""
    _on_gpu("x", x)
    dt = _dtype(x.dtype)
    px, ldx = _rows("x", x, None, None, x.dtype)
    pc, ps, pf, outputs = _grouped(codes, scales, offsets, x.shape[1], group, x.dtype, x)
    po, ldo = _rows("out", out, x.shape[0], outputs, x.dtype, x)
    _call(x, "sdnn_grouped_linear", px, ldx, dt, pc, ps, pf, x.shape[0], outputs, x.shape[1], group, po, ldo, *_workspace(workspace, x), _stream_handle(stream))
