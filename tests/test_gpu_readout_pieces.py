"""The readout where its classes or rows are gone over in more than one piece."""
import pytest

from tests.gpu_util import log
from tests.test_gpu_readout import Case, reference, assert_within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,classes,features", [(2048, 33068, 512), (4096, 16484, 200), (300, 700, 200), (100, 3000, 130), (3, 900, 100), (2100, 2100, 1030)])
def test_certain_answers_have_no_gradient(rows, classes, features, dtype):
    """Rows that answer their label with logits of 1e6 and more, far ahead of every other: exp(l - lse) is one to the bit, so
    dx and dw are zeros, wherever the label lies among the pieces of the classes (the last one may be small)."""
    log(f"readout certain {rows} x {classes} x {features} {dtype}")
    c = Case(rows, classes, features, dtype, seed=8)
    t = c.torch
    if rows > 100:
        c.y[: rows // 2] = t.randint(max(0, classes - 90), classes, (rows // 2,), device="cuda")
    c.x.copy_(1e6 * c.w[c.y].float())
    l = c.x.float() @ c.w.float().t()
    two = l.topk(2, 1).values
    assert t.equal(l.argmax(1), c.y) and float((two[:, 0] - two[:, 1]).min()) > 1e4
    c.run()
    assert not c.loss.any() and not c.dx.any() and not c.dw.any()


@pytest.mark.parametrize("dtype,rows,classes,features", [("bfloat16", 16384, 8192, 64), ("float32", 16384, 8192, 40)])
def test_dx_over_pieces_in_one_launch_each(dtype, rows, classes, features):
    """Blocks for all CUs, so dx's k is not split: the last piece's products finish the sums of the pieces before."""
    log(f"readout pieces, dx unsplit {dtype}")
    c = Case(rows, classes, features, dtype, seed=10)
    c.y[::9] = -1
    c.run()
    want = reference(c.torch, c.x, c.w, c.y, None)
    assert_within("dx", c.dx, want[2])
    assert_within("dw", c.dw, want[3])
