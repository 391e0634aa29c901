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


def sampled(c, some):
    """loss and lse of the rows `some` and their bounds, as if they were all."""
    t = c.torch
    x = c.x[some]
    want = reference(t, x, c.w, c.y[some], None)
    assert_within("loss", c.loss[some], want[0])
    live = (c.y[some] >= 0) & (c.y[some] < c.w.shape[0])
    assert_within("lse", c.lse[some][live], tuple(v[live] for v in want[1]))


class LossOnly(Case):
    def __init__(self, rows, classes, features, dtype, seed):
        from paper_1909_05631_amd import readout
        from tests.gpu_util import torch_cuda
        self.torch = torch = torch_cuda()
        gen = torch.Generator("cuda").manual_seed(seed)
        dt = getattr(torch, dtype)
        self.x = torch.randn(rows, features, generator=gen, device="cuda", dtype=torch.float32).to(dt)
        self.w = (torch.randn(classes, features, generator=gen, device="cuda") / features ** 0.5).to(dt)
        self.y = torch.randint(-1, classes + 1, (rows,), generator=gen, device="cuda")
        self.loss, self.lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
        ws = torch.full((readout.workspace_bytes(rows, classes, features, dt, gradient=False),), 255, dtype=torch.uint8, device="cuda")
        readout.loss(self.x, self.w, self.y, self.loss, self.lse, ws)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,classes,features", [(40000, 70001, 32), (300001, 4000, 48), (700, 1600003, 16)])
def test_loss_in_panels(rows, classes, features, dtype):
    """More than 2^30 logits: rows and classes in panels, the last of each ragged; labels of every panel, and none."""
    log(f"readout panels {rows} x {classes} x {features} {dtype}")
    c = LossOnly(rows, classes, features, dtype, 13)
    some = c.torch.cat([c.torch.arange(40), c.torch.arange(16380, 16390) % rows, c.torch.arange(rows - 40, rows), c.torch.randint(0, rows, (100,))]).cuda()
    sampled(c, some)
    out = (c.y < 0) | (c.y >= classes)
    assert not c.loss[out].any() and bool(c.loss.isfinite().all()) and bool((c.loss >= 0).all())


def test_loss_in_panels_of_infinities_and_nan():
    """What a row holds stays its own from panel to panel; a class of NaN makes NaN of every row."""
    log("readout panels, infinities")
    c = LossOnly(17000, 66000, 32, "bfloat16", 14)
    t, r = c.torch, __import__("paper_1909_05631_amd.readout", fromlist=["loss"])
    before, good = c.loss.clone(), (c.y >= 0) & (c.y < 66000)
    bad = t.nonzero(good)[[0, 5, -1], 0]
    c.x[bad[0], 3], c.x[bad[1], 0], c.x[bad[2], 1] = float("inf"), float("nan"), -float("inf")
    ws = t.empty(r.workspace_bytes(17000, 66000, 32, t.bfloat16, gradient=False), dtype=t.uint8, device="cuda")
    r.loss(c.x, c.w, c.y, c.loss, c.lse, ws)
    others = t.ones_like(good)
    others[bad] = False
    assert bool(c.loss[bad].isnan().all()) and t.equal(c.loss[others], before[others])
    for v in (100, 65900):
        w = c.w.clone()
        w[v, 2] = float("nan")
        r.loss(c.x, w, c.y, c.loss, c.lse, ws)
        assert bool(c.loss[good].isnan().all()) and not c.loss[~good].any()


def test_the_most_rows():
    """2^24 rows against 33000 classes, sizes that one launch of blocks cannot take."""
    log("readout 2^24 rows")
    c = LossOnly(1 << 24, 33000, 16, "bfloat16", 15)
    sampled(c, c.torch.randint(0, 1 << 24, (400,), device="cuda"))
    assert bool(c.loss.isfinite().all())
