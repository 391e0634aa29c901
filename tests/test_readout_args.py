"""The dense readout's entry points without a GPU: malformed arguments are refused on the host, by the C ABI with a
status and a message, by the binding with an exception, before any device is touched."""
import ctypes
import os

import pytest
import torch

from paper_1909_05631_amd import readout, sdnn

A = 1 << 20  # an aligned address that no call may follow


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sdnn.library_path()):
        from paper_1909_05631_amd import build
        build.build()
    return sdnn.load_library()


def refused(lib, status, message, fn, *args):
    assert fn(*args) == status
    assert message in lib.sdnn_last_error().decode()


def loss_args(**kw):
    a = dict(x=A, ldx=64, w=A, ldw=64, dtype=0, labels=A, rows=4, classes=10, features=64, loss=A, lse=A, ws=A, ws_bytes=1 << 30, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


def grad_args(**kw):
    a = dict(x=A, ldx=64, w=A, ldw=64, dtype=0, labels=A, lse=A, row_grad=None, rows=4, classes=10, features=64, dx=A, lddx=64, dw=A, lddw=64, ws=A,
             ws_bytes=1 << 30, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


@pytest.mark.parametrize("kw,status,message", [
    (dict(rows=-1), 1, "n_rows"), (dict(rows=(1 << 24) + 1), 1, "n_rows"), (dict(classes=0), 1, "n_classes"), (dict(classes=(1 << 24) + 1), 1, "n_classes"),
    (dict(features=0), 1, "n_features"), (dict(features=(1 << 20) + 1), 1, "n_features"), (dict(dtype=2), 1, "dtype"), (dict(dtype=-1), 1, "dtype"),
    (dict(x=None), 1, "x is null"), (dict(w=None), 1, "w is null"), (dict(x=A + 2), 1, "x is not aligned"), (dict(dtype=1, w=A + 1), 1, "w is not aligned"),
    (dict(ldx=63), 1, "row stride of x"), (dict(ldw=63), 1, "row stride of w"), (dict(labels=None), 1, "null"),
    (dict(ws_bytes=16), 5, "needed"), (dict(ws=None), 1, "workspace"), (dict(ws=A + 128), 1, "workspace"),
])
def test_loss_and_gradient_refuse(lib, kw, status, message):
    refused(lib, status, message, lib.sdnn_readout_loss, *loss_args(**kw))
    refused(lib, status, message, lib.sdnn_readout_grad, *grad_args(**kw))


def test_loss_refuses_no_loss_and_gradient_its_own(lib):
    refused(lib, 1, "loss is null", lib.sdnn_readout_loss, *loss_args(loss=None))
    refused(lib, 1, "null", lib.sdnn_readout_grad, *grad_args(lse=None))
    refused(lib, 1, "row stride of dx", lib.sdnn_readout_grad, *grad_args(lddx=1))
    refused(lib, 1, "row stride of dw", lib.sdnn_readout_grad, *grad_args(lddw=1))
    refused(lib, 1, "dw is not aligned", lib.sdnn_readout_grad, *grad_args(dw=A + 1))


def test_nothing_to_do_is_no_error(lib):
    assert lib.sdnn_readout_loss(*loss_args(rows=0, x=None, w=None, labels=None, loss=None, ws=None, ws_bytes=0)) == 0
    assert lib.sdnn_readout_grad(*grad_args(dx=None, dw=None)) == 0
    assert lib.sdnn_readout_grad(*grad_args(rows=0, dw=None)) == 0
    assert lib.sdnn_mx_quantize(None, 0, 0, 0, 32, None, None, None) == 0
    assert lib.sdnn_mx_product(None, None, None, None, 0, 5, 32, None, 0, 0, None) == 0
    assert lib.sdnn_mx_product(None, None, None, None, 5, 0, 32, None, 0, 0, None) == 0
    coef = (ctypes.c_float * 3)(1, 1, 1)
    assert lib.sdnn_orthogonalize(None, 0, 0, None, 0, 0, 0, 0, 4, 4, 5, coef, 0.0, None, 0, None) == 0


def test_workspace_sizes(lib):
    f = lib.sdnn_readout_workspace_bytes
    for bad in ((-1, 1, 1, 0), (1, 0, 1, 0), (1, 1, 0, 0), (1, 1, 1, 7)):
        assert f(*bad, 0) == 0 and f(*bad, 1) == 0
    assert 0 < f(100, 1000, 64, 1, 0) <= f(100, 1000, 64, 1, 1)
    # the logits of all rows and classes are never there: 2^13 x 2^17 of them would be 4 GiB in fp32
    assert f(1 << 13, 1 << 17, 64, 1, 1) < 1 << 30
    assert lib.sdnn_orthogonalize_workspace_bytes(1, 0, 5) == 0 and lib.sdnn_orthogonalize_workspace_bytes(65536, 5, 5) == 0
    assert lib.sdnn_orthogonalize_workspace_bytes(2, 30, 50) > 2 * 30 * 50 * 8
    assert lib.sdnn_mx_linear_workspace_bytes(-1, 32) == 0 and lib.sdnn_mx_linear_workspace_bytes(3, 100) >= 3 * 68
    assert [lib.sdnn_mx_blocks(n) for n in (0, 1, 32, 128, 129, 1000)] == [0, 4, 4, 4, 8, 32]


def orth_args(**kw):
    a = dict(g=A, ldg=64, bg=4096, out=A, ldo=64, bo=4096, dtype=0, batch=2, rows=64, cols=64, steps=5, coef=(ctypes.c_float * 3)(3.4, -4.7, 2.0), eps=1e-7,
             ws=A, ws_bytes=1 << 30, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


@pytest.mark.parametrize("kw,status,message", [
    (dict(batch=-1), 1, "batch"), (dict(batch=65536), 1, "batch"), (dict(rows=0), 1, "rows"), (dict(cols=0), 1, "cols"), (dict(cols=(1 << 20) + 1), 1, "cols"),
    (dict(dtype=3), 1, "dtype"), (dict(steps=-1), 1, "steps"), (dict(steps=33), 1, "steps"), (dict(coef=None), 1, "coefficients"),
    (dict(coef=(ctypes.c_float * 3)(1, float("nan"), 1)), 1, "coefficient 1"), (dict(coef=(ctypes.c_float * 3)(1, 1, float("inf"))), 1, "coefficient 2"),
    (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"), (dict(g=None), 1, "g is null"), (dict(out=None), 1, "out is null"),
    (dict(ldg=63), 1, "row stride of g"), (dict(ldo=63), 1, "row stride of out"), (dict(bo=4095), 1, "batch stride"), (dict(bg=-1), 1, "batch stride"),
    (dict(ws_bytes=1), 5, "needed"), (dict(ws=A + 8), 1, "workspace"),
])
def test_orthogonalize_refuses(lib, kw, status, message):
    refused(lib, status, message, lib.sdnn_orthogonalize, *orth_args(**kw))


def test_mx_refuses(lib):
    q, d, p, l = lib.sdnn_mx_quantize, lib.sdnn_mx_dequantize, lib.sdnn_mx_product, lib.sdnn_mx_linear
    refused(lib, 1, "n_rows", q, A, 64, 0, -1, 64, A, A, None)
    refused(lib, 1, "n_values", q, A, 64, 0, 1, 0, A, A, None)
    refused(lib, 1, "dtype", q, A, 64, 9, 1, 64, A, A, None)
    refused(lib, 1, "row stride of x", q, A, 63, 0, 1, 64, A, A, None)
    refused(lib, 1, "codes", q, A, 64, 0, 1, 64, A + 8, A, None)
    refused(lib, 1, "scales", q, A, 64, 0, 1, 64, A, A + 2, None)
    refused(lib, 1, "null", q, A, 64, 0, 1, 64, None, A, None)
    refused(lib, 1, "out is null", d, A, A, 1, 64, None, 64, 0, None)
    refused(lib, 1, "null", d, A, None, 1, 64, A, 64, 0, None)
    refused(lib, 1, "n_outputs", p, A, A, A, A, 1, -1, 64, A, 64, 0, None)
    refused(lib, 1, "row stride of out", p, A, A, A, A, 1, 65, 64, A, 64, 0, None)
    refused(lib, 1, "codes or scales of w", p, A, A, None, A, 1, 64, 64, A, 64, 0, None)
    refused(lib, 5, "needed", l, A, 64, 0, A, A, 1, 64, 64, A, 64, A, 1, None)
    refused(lib, 1, "workspace", l, A, 64, 0, A, A, 1, 64, 64, A, 64, None, 1 << 20, None)
    refused(lib, 1, "row stride of x", l, A, 63, 0, A, A, 1, 64, 64, A, 64, A, 1 << 20, None)


def test_binding_refuses_tensors_off_the_gpu():
    x, y = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: readout.loss(x, x, y, x[:, 0], None, x), lambda: readout.gradient(x, x, y, x[:, 0], x, x, x), lambda: readout.orthogonalize(x, x, x),
                 lambda: readout.mx_quantize(x, x, x), lambda: readout.mx_dequantize(x, x, x), lambda: readout.mx_product(x, x, x, x, 8, x),
                 lambda: readout.mx_linear(x, x, x, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="float16"):
        readout.workspace_bytes(1, 1, 1, torch.float16)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes", [(60000, 65536), (60000, 131072), (1 << 20, 65536), (1 << 22, 1 << 18), (1000, 1 << 24), (1 << 24, 1 << 15)])
def test_workspace_does_not_grow_with_rows_times_classes(lib, rows, classes, dtype):
    """Past what grows with the rows (at most 8 bytes a value of x, and 40 a row) and with the classes (the same), the loss takes at
    most 256 MB and 1 MB of rounding; the gradient, with sums of dx and parts of 6 bytes a value too, 6 bytes times its
    values of G."""
    f, d = lib.sdnn_readout_workspace_bytes, 64
    assert f(rows, classes, d, dtype, 0) <= (rows + classes) * (8 * d + 40) + (257 << 20)
    splits = 64  # parts of k whose sums may be kept
    assert f(rows, classes, d, dtype, 1) <= (rows + classes) * ((14 + 4) * d + 40) + splits * 4 * d * min(rows, classes) + 6 * max(1 << 26, 256 * rows) + (257 << 20)


@pytest.mark.parametrize("coefficients", [(), (1.5, -0.5), (1.0, 1.0, 1.0, 1.0), 3.0, ("a", 1, 1)])
def test_binding_refuses_coefficients_that_are_not_three_numbers(coefficients):
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="coefficients"):
        readout.orthogonalize(x, x, x, coefficients=coefficients)
