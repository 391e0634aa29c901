"""The gated layer, the clipped gradients and the 4-bit weights with group scales without a GPU: malformed arguments are
refused on the host, by the C ABI with a status and a message, by the binding with an exception, before any device is
touched."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1909_05631_amd import readout
from tests.test_readout_args import A, lib, refused  # noqa: F401


def args(defaults, kw):
    assert set(kw) <= set(defaults)
    return list({**defaults, **kw}.values())


def layer_args(**kw):
    return args(dict(x=A, ldx=64, wg=A, ldwg=64, wu=A, ldwu=64, dtype=0, act=0, rows=4, hidden=10, features=64, h=A, ldh=10, gate=A, ldgate=10, up=A, ldup=10, ws=A, ws_bytes=1 << 30, stream=None), kw)


def grad_args(**kw):
    return args(dict(x=A, ldx=64, wg=A, ldwg=64, wu=A, ldwu=64, dtype=0, act=0, gate=A, ldgate=10, up=A, ldup=10, dh=A, lddh=10, rows=4, hidden=10, features=64, dx=A, lddx=64, dwg=A, lddwg=64, dwu=A,
                     lddwu=64, ws=A, ws_bytes=1 << 30, stream=None), kw)


@pytest.mark.parametrize("kw,status,message", [
    (dict(rows=-1), 1, "n_rows"), (dict(rows=(1 << 24) + 1), 1, "n_rows"), (dict(hidden=0), 1, "n_hidden"), (dict(hidden=(1 << 19) + 1), 1, "n_hidden"), (dict(features=0), 1, "n_features"),
    (dict(features=(1 << 20) + 1), 1, "n_features"), (dict(dtype=2), 1, "dtype"), (dict(dtype=-1), 1, "dtype"), (dict(act=3), 1, "activation"), (dict(act=-1), 1, "activation"),
    (dict(x=None), 1, "x is null"), (dict(wg=None), 1, "w_gate is null"), (dict(wu=None), 1, "w_up is null"), (dict(x=A + 2), 1, "x is not aligned"), (dict(dtype=1, wu=A + 1), 1, "w_up is not aligned"),
    (dict(ldx=63), 1, "row stride of x"), (dict(ldwg=63), 1, "row stride of w_gate"), (dict(ldwu=63), 1, "row stride of w_up"), (dict(ldgate=9), 1, "row stride of gate"),
    (dict(up=A + 1), 1, "up is not aligned"), (dict(ws_bytes=16), 5, "needed"), (dict(ws=None), 1, "workspace"), (dict(ws=A + 128), 1, "workspace"),
])
def test_layer_and_gradient_refuse(lib, kw, status, message):  # noqa: F811
    refused(lib, status, message, lib.sdnn_gated, *layer_args(**kw))
    refused(lib, status, message, lib.sdnn_gated_grad, *grad_args(**kw))


def test_layer_refuses_no_result_and_gradient_its_own(lib):  # noqa: F811
    refused(lib, 1, "h is null", lib.sdnn_gated, *layer_args(h=None))
    refused(lib, 1, "row stride of h", lib.sdnn_gated, *layer_args(ldh=9))
    refused(lib, 1, "dh is null", lib.sdnn_gated_grad, *grad_args(dh=None))
    refused(lib, 1, "together", lib.sdnn_gated_grad, *grad_args(up=None))
    refused(lib, 1, "together", lib.sdnn_gated_grad, *grad_args(gate=None))
    for name in ("dx", "dwg", "dwu"):
        refused(lib, 1, "row stride of d", lib.sdnn_gated_grad, *grad_args(**{"ld" + name: 63}))
    # without gate and up it needs room for them
    kept, again = (lib.sdnn_gated_workspace_bytes(4, 10, 64, 0, g) for g in (1, 2))
    assert kept < again
    refused(lib, 5, "needed", lib.sdnn_gated_grad, *grad_args(gate=None, up=None, ws_bytes=kept))


def test_nothing_to_do_is_no_error(lib):  # noqa: F811
    assert lib.sdnn_gated(*layer_args(rows=0, x=None, wg=None, wu=None, h=None, ws=None, ws_bytes=0)) == 0
    assert lib.sdnn_gated_grad(*grad_args(dx=None, dwg=None, dwu=None)) == 0
    assert lib.sdnn_gated_grad(*grad_args(rows=0, x=None, dh=None, dwg=None, dwu=None)) == 0
    assert lib.sdnn_grouped_quantize(None, 0, 0, 0, 32, 32, None, None, None, None) == 0
    assert lib.sdnn_grouped_dequantize(None, None, None, 0, 0, 32, 32, None, 0, None) == 0
    assert lib.sdnn_grouped_linear(*linear_args(rows=0, x=None, codes=None)) == 0
    assert lib.sdnn_grouped_linear(*linear_args(outputs=0, x=None, codes=None)) == 0


def test_workspace_sizes(lib):  # noqa: F811
    f = lib.sdnn_gated_workspace_bytes
    for bad in ((-1, 1, 1, 0), (1, 0, 1, 0), (1, 1, 0, 0), (1, 1, 1, 7), (1, (1 << 19) + 1, 1, 0)):
        assert [f(*bad, g) for g in range(3)] == [0, 0, 0]
    assert f(1, 1, 1, 0, 3) == 0 and f(1, 1, 1, 0, -1) == 0
    for sizes in ((1, 1, 1), (5, 300, 70), (1021, 2047, 1000), (8192, 16384, 4096), (1 << 24, 1, 1)):
        for dtype in (0, 1):
            layer, kept, again = (f(*sizes, dtype, g) for g in range(3))
            assert 0 < layer <= kept <= again
    g = lib.sdnn_clip_workspace_bytes
    assert g(-1) == 0 and g(4097) == 0 and 0 < g(0) <= g(1) <= g(4096) < 1 << 20
    h = lib.sdnn_grouped_linear_workspace_bytes
    assert h(-1, 5, 5, 0) == 0 and h(5, -1, 5, 0) == 0 and h(5, 5, 0, 0) == 0 and h(5, 5, 5, 2) == 0
    assert h(1, 1 << 24, 1 << 14, 1) == 0 and h(65, 100, 100, 1) > 0  # one row of x stays in LDS
    assert [lib.sdnn_grouped_groups(n, g) for n, g in ((0, 32), (1, 32), (32, 32), (33, 32), (1000, 64), (1 << 20, 128), ((1 << 20) + 1, 32), (5, 16))] == [0, 1, 1, 2, 16, 8192, 0, 0]
    assert [readout.grouped_groups(n, g) for n, g in ((0, 32), (1, 32), (33, 32), (1000, 64), (5, 16))] == [0, 1, 2, 16, 0]


def tensors(*rows):
    """A list of sdnn_tensor: data, out, rows, cols, ld, ldo, dtype."""
    table = np.array(rows, np.int64).reshape(-1, 7)
    return table, table.ctypes.data


GOOD = (A, 0, 3, 8, 8, 0, 0)


@pytest.mark.parametrize("row,message", [
    ((0, 0, 3, 8, 8, 0, 0), "null"), ((A + 2, 0, 3, 8, 8, 0, 0), "aligned"), ((A + 1, 0, 3, 8, 8, 0, 1), "aligned"), ((A, 0, 3, 8, 8, 0, 2), "dtype"), ((A, 0, -1, 8, 8, 0, 0), "outside"),
    ((A, 0, 3, -8, 8, 0, 0), "outside"), ((A, 0, 1 << 21, 1 << 20, 1 << 20, 0, 0), "outside"), ((A, 0, 3, 8, 7, 0, 0), "row stride"),
])
def test_lists_refuse(lib, row, message):  # noqa: F811
    table, at = tensors(GOOD, row)
    for call in (lambda: lib.sdnn_global_norm(at, 2, A, A, 1 << 20, None), lambda: lib.sdnn_clip(at, 2, 1.0, A, A, 1 << 20, None)):
        assert call() == 1
        assert message in lib.sdnn_last_error().decode() and "tensor 1" in lib.sdnn_last_error().decode()


def test_clip_refuses(lib):  # noqa: F811
    f = lib.sdnn_clip
    table, at = tensors(GOOD, (A + 4096, 0, 3, 8, 8, 0, 0))
    refused(lib, 1, "n_tensors", f, at, -1, 1.0, A, A, 1 << 20, None)
    refused(lib, 1, "n_tensors", f, at, 4097, 1.0, A, A, 1 << 20, None)
    refused(lib, 1, "tensors is null", f, None, 2, 1.0, A, A, 1 << 20, None)
    refused(lib, 1, "max_norm", f, at, 2, -0.5, A, A, 1 << 20, None)
    refused(lib, 1, "max_norm", f, at, 2, float("nan"), A, A, 1 << 20, None)
    refused(lib, 1, "norm", f, at, 2, 1.0, None, A, 1 << 20, None)
    refused(lib, 1, "norm", f, at, 2, 1.0, A + 2, A, 1 << 20, None)
    refused(lib, 5, "needed", f, at, 2, 1.0, A, A, 64, None)
    refused(lib, 1, "workspace", f, at, 2, 1.0, A, A + 8, 1 << 20, None)
    refused(lib, 1, "norm", lib.sdnn_global_norm, at, 2, None, A, 1 << 20, None)
    for row, message in (((A, A + 2, 3, 8, 8, 8, 0), "out is not aligned"), ((A, A + 64, 3, 8, 8, 7, 0), "row stride of out"), ((A, A, 3, 8, 9, 8, 0), "another row stride")):
        bad, to = tensors(row)
        refused(lib, 1, message, f, to, 1, 1.0, A, A, 1 << 20, None)


@pytest.mark.parametrize("n", [2, 17, 300, 4096])
def test_two_tensors_written_to_one_place_are_refused(lib, n):  # noqa: F811
    """Wherever in the list they stand, in place and apart; empty ones do not count. (The workspace is refused later: nothing
    is enqueued for a list without fault either.)"""
    rows = [(A + 4096 * i, 0, 3, 8, 8, 0, 0) for i in range(n)]
    for i, j in ((0, 1), (0, n - 1), (n // 2 - 1, n // 2)):
        if i == j:
            continue
        bad = list(rows)
        bad[j] = (A + (1 << 30), rows[i][0], 3, 8, 8, 8, 0)
        table, at = tensors(*bad)
        refused(lib, 1, f"tensors {i} and {j} are written", lib.sdnn_clip, at, n, 1.0, A, A, 1 << 24, None)
        bad[j] = (rows[i][0], 0, 0, 8, 8, 0, 0)
        table, at = tensors(*bad)
        refused(lib, 5, "needed", lib.sdnn_clip, at, n, 1.0, A, A, 64, None)


def linear_args(**kw):
    return args(dict(x=A, ldx=64, dtype=0, codes=A, scales=A, offsets=None, rows=4, outputs=10, n=64, group=32, out=A, ldo=10, ws=A, ws_bytes=1 << 30, stream=None), kw)


@pytest.mark.parametrize("kw,status,message", [
    (dict(rows=-1), 1, "n_rows"), (dict(rows=(1 << 24) + 1), 1, "n_rows"), (dict(n=0), 1, "n_values"), (dict(n=(1 << 20) + 1), 1, "n_values"), (dict(group=0), 1, "group"), (dict(group=48), 1, "group"),
    (dict(group=256), 1, "group"), (dict(dtype=2), 1, "dtype"), (dict(outputs=-1), 1, "n_outputs"), (dict(outputs=(1 << 24) + 1), 1, "n_outputs"), (dict(x=None), 1, "x is null"), (dict(ldx=63), 1, "row stride of x"),
    (dict(codes=None), 1, "null"), (dict(scales=None), 1, "null"), (dict(codes=A + 8), 1, "codes are not"), (dict(scales=A + 2), 1, "scales or offsets"), (dict(offsets=A + 2), 1, "scales or offsets"),
    (dict(out=None), 1, "out is null"), (dict(ldo=9), 1, "row stride of out"), (dict(rows=65, ws_bytes=16), 5, "needed"), (dict(rows=65, ws=None), 1, "workspace"), (dict(rows=65, ws=A + 8), 1, "workspace"),
])
def test_linear_refuses(lib, kw, status, message):  # noqa: F811
    refused(lib, status, message, lib.sdnn_grouped_linear, *linear_args(**kw))


def test_quantize_and_dequantize_refuse(lib):  # noqa: F811
    q, d = lib.sdnn_grouped_quantize, lib.sdnn_grouped_dequantize
    refused(lib, 1, "n_rows", q, A, 64, 0, -1, 64, 32, A, A, None, None)
    refused(lib, 1, "n_values", q, A, 64, 0, 1, 0, 32, A, A, None, None)
    refused(lib, 1, "group", q, A, 64, 0, 1, 64, 33, A, A, None, None)
    refused(lib, 1, "row stride of w", q, A, 63, 0, 1, 64, 32, A, A, None, None)
    refused(lib, 1, "w is null", q, None, 64, 0, 1, 64, 32, A, A, None, None)
    refused(lib, 1, "codes", q, A, 64, 0, 1, 64, 32, A + 4, A, None, None)
    refused(lib, 1, "null", q, A, 64, 0, 1, 64, 32, A, None, None, None)
    refused(lib, 1, "offsets", q, A, 64, 1, 1, 64, 32, A, A, A + 1, None)
    refused(lib, 1, "out is null", d, A, A, None, 0, 1, 64, 32, None, 64, None)
    refused(lib, 1, "row stride of out", d, A, A, None, 0, 1, 64, 32, A, 63, None)
    refused(lib, 1, "dtype", d, A, A, None, 5, 1, 64, 32, A, 64, None)


def test_binding_refuses_tensors_off_the_gpu():
    x, b = torch.zeros(4, 64), torch.zeros(4, 32, dtype=torch.uint8)
    for call in (lambda: readout.gated(x, x, x, x, x), lambda: readout.gated_gradient(x, x, x, x, x, x, x, x), lambda: readout.global_norm([x], x, x), lambda: readout.clip([x], 1.0, x, x),
                 lambda: readout.grouped_quantize(x, b, x), lambda: readout.grouped_dequantize(b, x, x), lambda: readout.grouped_linear(x, b, x, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="float16"):
        readout.gated_workspace_bytes(1, 1, 1, torch.float16)
    with pytest.raises(ValueError, match="float64"):
        readout.grouped_linear_workspace_bytes(1, 1, 1, torch.float64)
    with pytest.raises(ValueError, match="tanh"):
        readout.gated(x, x, x, x, x, activation="tanh")


def test_list_entries_are_as_the_header_has_them():
    """The binding writes sdnn_tensor as seven words: two addresses, four 64-bit sizes, a 32-bit type in the low half."""
    class Tensor(ctypes.Structure):
        _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("ldo", ctypes.c_int64), ("dtype", ctypes.c_int32)]
    assert ctypes.sizeof(Tensor) == 56 and [getattr(Tensor, n).offset for n, _ in Tensor._fields_] == [0, 8, 16, 24, 32, 40, 48]
