"""The dense readout's operators on the GPU against plain evaluations in 64 bits.

Bounds. u16 = 2^-8 and u32 = 2^-24 are the unit roundoffs of bf16 and fp32. A sum of k products in fp32, in
any order of the matrix instructions (32 products each, at most 3 per product for fp32 inputs), is off by at most
s(k) = (3 k / 32 + 40) u32 times the sum of magnitudes; products of fp32 inputs held in two fp16 parts add 4 * 2^-22 times it
(each part is cut at 2^-22, low times low is left out), and 2^-38 k times the largest magnitudes (what the parts cannot
hold). From the logits' bound d: lse and loss are within 2 d and a few u32 of their sizes, the probabilities within
a relative 4 d + (|l - lse| + 8) 2^-22 (exp's argument and result), and the products of G follow the same rules, with u16
for G's own rounding where the inputs are bf16, and u16 or u32 for the output's."""
import math

import numpy as np
import pytest

from tests.gpu_util import log, torch_cuda

pytestmark = pytest.mark.gpu
U16, U32 = 2.0 ** -8, 2.0 ** -24


def sum_bound(k):
    return (3 * k / 32 + 40) * U32


def product_bound(a, b, fp32):
    """Elementwise bound of the error of a b^T (rows of a, rows of b)."""
    k = a.shape[1]
    e = (sum_bound(k) + (4 * 2.0 ** -22 if fp32 else 0)) * (a.abs() @ b.abs().t())
    return e + 2.0 ** -38 * k * a.abs().max() * b.abs().max() if fp32 else e


def reference(torch, x, w, y, g):
    """loss, lse, dx, dw in 64 bits and the bounds of what the library's may be off."""
    fp32 = x.dtype == torch.float32
    classes = w.shape[0]
    live = (y >= 0) & (y < classes)
    x, w = x.double(), w.double()
    x = torch.where(live[:, None], x, 0.0)  # rows without a label count as zeros: nothing may depend on them
    l = x @ w.t()
    d = product_bound(x, w, fp32)
    top = d.max(1).values
    lse = torch.logsumexp(l, 1)
    at = y.clamp(0, classes - 1)[:, None]
    picked = l.gather(1, at)[:, 0]
    loss = torch.where(live, lse - picked, 0.0)
    few = 16 * U32 * (1 + lse.abs() + picked.abs() + math.log(classes))
    if g is None:
        g = torch.full_like(lse, 1.0 / max(1, int(live.sum())))
    g = torch.where(live, g.double(), 0.0)
    p = torch.exp(l - lse[:, None])
    ep = p * (4 * top[:, None] + (l.sub(lse[:, None]).abs() + 8) * 2.0 ** -22 + 4 * few[:, None]) + 2.0 ** -23
    G = p.scatter_add(1, at, -torch.ones_like(at, dtype=torch.float64)) * g[:, None]
    eG = ep * g[:, None].abs()
    eG += (2.0 ** -22 if fp32 else U16) * (G.abs() + eG) + (2.0 ** -39 * g.abs().max() if fp32 else 0)
    u = U32 if fp32 else U16
    dx, dw = G @ w, G.t() @ x
    bx = eG @ w.abs() + product_bound(G, w.t(), fp32)
    bw = eG.t() @ x.abs() + product_bound(G.t(), x.t(), fp32)
    bx, bw = (b + 4 * u * (r.abs() + b) for b, r in ((bx, dx), (bw, dw)))
    return (loss, 2 * top + few), (lse, top + few), (dx, bx), (dw, bw)


def assert_within(name, got, want):
    value, bound = want
    got = got.double()
    assert bool(got.isfinite().all()), f"{name} is not finite"
    over = ((got - value).abs() - bound).max()
    assert float(over) <= 1e-30, f"{name} is {float(over):.3g} over its bound"


def matrix(torch, gen, rows, cols, dtype, scale=1.0, pad=0, offset=0):
    """A matrix whose rows are `pad` values apart and whose first value lies `offset` values into its memory; what
    surrounds it is NaN."""
    flat = torch.full((rows * (cols + pad) + offset + pad + 8,), float("nan"), dtype=dtype, device="cuda")
    m = torch.as_strided(flat, (rows, cols), (cols + pad, 1), offset)
    m.copy_((torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dtype))
    return m


class Case:
    def __init__(self, rows, classes, features, dtype, seed=0, pad=0, offset=0, positive=True):
        from paper_1909_05631_amd import readout
        self.torch = torch = torch_cuda()
        self.r = readout
        gen = torch.Generator("cuda").manual_seed(seed)
        dt = getattr(torch, dtype)
        self.x = matrix(torch, gen, rows, features, dt, 1.0, pad, offset)
        if positive:
            self.x.clamp_(min=0)
        self.w = matrix(torch, gen, classes, features, dt, 1.5 / math.sqrt(features), pad, offset)
        self.y = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
        self.loss, self.lse = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
        self.dx, self.dw = (matrix(torch, gen, *t.shape, dt, 1.0, pad, offset).fill_(7) for t in (self.x, self.w))
        self.ws = torch.full((readout.workspace_bytes(rows, classes, features, dt),), 255, dtype=torch.uint8, device="cuda")

    def run(self, g=None, stream=None):
        self.r.loss(self.x, self.w, self.y, self.loss, self.lse, self.ws, stream=stream)
        self.r.gradient(self.x, self.w, self.y, self.lse, self.dx, self.dw, self.ws, row_grad=g, stream=stream)

    def check(self, g=None):
        want = reference(self.torch, self.x, self.w, self.y, g)
        live = (self.y >= 0) & (self.y < self.w.shape[0])
        assert_within("loss", self.loss, want[0])
        assert_within("lse", self.lse[live], tuple(t[live] for t in want[1]))
        assert_within("dx", self.dx, want[2])
        assert_within("dw", self.dw, want[3])


SHAPES = [(1, 1, 1), (1, 10, 64), (2, 2, 3), (5, 33, 31), (17, 129, 65), (64, 256, 128), (100, 10, 1024), (257, 1000, 72), (300, 4099, 40), (1021, 130, 500),
          (3, 20000, 64), (2500, 300, 33)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,classes,features", SHAPES)
def test_loss_and_gradient(rows, classes, features, dtype):
    log(f"readout {rows} x {classes} x {features} {dtype}")
    c = Case(rows, classes, features, dtype, seed=rows)
    c.run()
    c.check()
    g = c.torch.randn(rows, generator=c.torch.Generator("cuda").manual_seed(1), device="cuda")
    c.run(g)
    c.check(g)


# few rows, few classes (both sides of what they take), features past one, four and sixteen steps of a workgroup's columns
FEW = [(1, 300, 1024), (1, 301, 1025), (1, 70, 4097), (1, 33, 16384), (1, 33, 16385), (2, 1000, 1000), (3, 50, 1030), (4, 40, 4096), (4, 40, 4097), (5, 77, 1024), (16, 513, 1023),
       (16, 30, 1025), (17, 30, 100), (500, 16, 1024), (301, 2, 4000), (77, 1, 9001), (40, 1, 64), (1300, 3, 65), (9, 9, 9), (2, 3000, 5000)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,classes,features", FEW)
def test_few_rows_and_few_classes(rows, classes, features, dtype):
    log(f"readout few {rows} x {classes} x {features} {dtype}")
    c = Case(rows, classes, features, dtype, seed=classes, pad=rows % 3, offset=rows % 2)
    if rows > 3:
        c.y[1], c.y[3] = -1, classes
        c.x[1] = float("nan")
    c.run()
    c.check()
    g = c.torch.randn(rows, generator=c.torch.Generator("cuda").manual_seed(1), device="cuda")
    c.run(g)
    c.check(g)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (8, 0), (3, 5), (24, 8)])
def test_strides_and_alignment(pad, offset, dtype):
    """Rows apart from each other, bases on any value, NaN all around: nothing outside a matrix is used or written."""
    log(f"readout strides {pad} {offset} {dtype}")
    for rows, classes, features in ((70, 140, 96), (70, 140, 97)):
        c = Case(rows, classes, features, dtype, seed=3, pad=pad, offset=offset)
        around = [t.as_strided((t.untyped_storage().nbytes() // t.element_size(),), (1,), 0) for t in (c.dx, c.dw)]
        before = [a.isnan().sum() for a in around]
        c.run()
        c.check()
        assert [a.isnan().sum() for a in around] == before


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_without_a_label(dtype):
    """They hold NaN, infinities and huge values; labels are below, at and past the ends."""
    log(f"readout masked rows {dtype}")
    c = Case(150, 70, 64, dtype, seed=5)
    t = c.torch
    out = t.tensor([0, 3, 64, 65, 100, 149], device="cuda")
    c.y[out] = t.tensor([-1, 70, -100, 1 << 40, -(1 << 62), 71], device="cuda")
    c.x[0], c.x[3, 5], c.x[64], c.x[65, 0], c.x[100] = float("nan"), float("inf"), -float("inf"), 3e38, 1e30
    g = t.rand(150, device="cuda")
    g[out] = float("nan")
    for weights in (None, g):
        c.run(weights)
        c.check(None if weights is None else weights)
        assert not c.loss[out].any() and not c.dx[out].any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_row_has_a_label(dtype):
    log(f"readout all masked {dtype}")
    c = Case(33, 9, 40, dtype)
    c.y.fill_(-1)
    c.x.fill_(float("nan"))
    c.run()
    assert not c.loss.any() and not c.dx.any() and not c.dw.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_rows(dtype):
    log(f"readout no rows {dtype}")
    c = Case(0, 9, 40, dtype)
    c.run()
    assert not c.dw.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_several_pieces(dtype):
    """More classes than one piece of G holds (2^26 values): dx adds up over the pieces, the last one ragged."""
    log(f"readout pieces {dtype}")
    c = Case(2048, 40001, 72, dtype, seed=9)
    c.y[::7] = -1
    c.run()
    c.check()


def test_wide_range():
    """fp32 rows of very different sizes, weights likewise; exponentials that vanish; a certain answer."""
    log("readout wide range")
    c = Case(64, 50, 128, "float32", seed=2)
    t = c.torch
    c.x *= t.exp2(t.arange(64, device="cuda") % 23 - 16.0)[:, None]
    c.w *= t.exp2(t.arange(50, device="cuda") % 9 - 4.0)[:, None]
    c.run()
    c.check()


def test_equal_weights_cost_no_precision():
    """bf16, every row's weight the same and halfway between two bf16 values: a weight rounded by itself would move every
    gradient by u16. G's and the output's own roundings are independent, each at most 0.5 u16 on average over a binade in
    the root mean square, so together under 0.75 u16."""
    log("readout equal weights")
    c = Case(400, 500, 256, "bfloat16", seed=12)
    g = c.torch.full((400,), 1.0 + 0.999 * U16 / 2, device="cuda")
    c.run(g)
    c.check(g)
    _, _, dx, dw = reference(c.torch, c.x, c.w, c.y, g)
    for got, want in ((c.dx, dx[0]), (c.dw, dw[0])):
        assert float((got.double() - want).norm() / want.norm()) <= 0.75 * U16


@pytest.mark.parametrize("what", ["dx", "dw"])
def test_one_gradient_alone(what):
    log(f"readout {what} alone")
    c = Case(90, 50, 64, "float32")
    c.run()
    want = getattr(c, what).clone()
    getattr(c, what).fill_(5)
    other = "dw" if what == "dx" else "dx"
    kept = getattr(c, other).clone()
    args = {"dx": None, "dw": None, what: getattr(c, what)}
    c.r.gradient(c.x, c.w, c.y, c.lse, args["dx"], args["dw"], c.ws)
    assert c.torch.equal(getattr(c, what), want) and c.torch.equal(getattr(c, other), kept)


def test_gradient_against_differences():
    """Directional derivatives of the loss as the library computes it: (L(x + h d) - L(x - h d)) / 2h. The loss's error is at
    most 1e-5 a row (its bound, with |l| < 16), that of the difference quotient h^2 / 6 times the third derivative along d, at
    most max |l'|^3 with |l'| the logits' change along d."""
    log("readout differences")
    c = Case(40, 30, 64, "float32", seed=11)
    t = c.torch
    c.run()
    h = 0.02
    gen = t.Generator("cuda").manual_seed(4)
    for name, grad in (("x", c.dx), ("w", c.dw)):
        base = getattr(c, name).clone()
        d = t.randn(base.shape, generator=gen, device="cuda")
        d /= d.norm(dim=1, keepdim=True)
        total = []
        for sign in (1, -1):
            getattr(c, name).copy_(base + sign * h * d)
            c.r.loss(c.x, c.w, c.y, c.loss, None, c.ws)
            total.append(float(c.loss.double().mean()))
        getattr(c, name).copy_(base)
        along = (d.double() @ c.w.double().t() if name == "x" else c.x.double() @ d.double().t()).abs().max()
        want = float((grad.double() * d.double()).sum())
        assert abs((total[0] - total[1]) / (2 * h) - want) <= 1e-5 / h + h * h / 6 * float(2 * along) ** 3


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_same_bits_on_any_stream_and_in_a_graph(dtype):
    log(f"readout streams and graph {dtype}")
    c = Case(300, 700, 200, dtype, seed=6)
    t = c.torch
    c.run()
    want = [v.clone() for v in (c.loss, c.lse, c.dx, c.dw)]
    side = t.cuda.Stream()
    busy = t.rand(4096, 4096, device="cuda")
    t.cuda.synchronize()
    for v in (c.loss, c.lse, c.dx, c.dw):
        v.fill_(3)
    side.wait_stream(t.cuda.current_stream())
    for _ in range(4):
        busy = busy @ busy * 1e-4
    c.run(stream=side)
    side.synchronize()
    assert all(t.equal(a, b) for a, b in zip((c.loss, c.lse, c.dx, c.dw), want))
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        c.run(stream=t.cuda.current_stream())
    for k in range(4):
        c.x.mul_(0.5 + 0.25 * k)
        graph.replay()
        t.cuda.synchronize()
        got = [v.clone() for v in (c.loss, c.lse, c.dx, c.dw)]
        for v in (c.loss, c.lse, c.dx, c.dw):
            v.fill_(3)
        c.run(stream=t.cuda.current_stream())
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip((c.loss, c.lse, c.dx, c.dw), got)), f"replay {k}"


# ------------------------------------------------------------------------------------------------

MUON = (3.4445, -4.7750, 2.0315)


def newton_schulz(torch, g, steps, coef, eps, dtype):
    a, b, c = coef
    x = g.to(dtype)
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for i in range(steps):
        xt = x.transpose(-2, -1).contiguous()
        m = torch.matmul(x, xt) if x.shape[-2] <= x.shape[-1] else torch.matmul(xt, x)
        k = b * m + c * torch.matmul(m, m)
        x = a * x + (torch.matmul(k, x) if x.shape[-2] <= x.shape[-1] else torch.matmul(x, k))
    return x


def orth_bound(g, out32, exact):
    """Rounding grows by at most |p'| <= 4 a step (singular values stay below 1.3), from 2^-20 a product; in practice far
    less, so a result is also held to 4 times what the same steps in fp32 lose."""
    plain = float((out32.double() - exact).norm())
    return 4 * plain + 4 * U32 * float(exact.norm())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (1, 1, 7), (1, 9, 1), (3, 16, 16), (2, 31, 65), (1, 64, 200), (2, 130, 64), (1, 257, 255), (1, 300, 700), (1, 700, 300),
                                             (5, 40, 1000), (1, 520, 520)])
def test_orthogonalize(batch, rows, cols, dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize {batch} x {rows} x {cols} {dtype}")
    gen = torch.Generator("cuda").manual_seed(rows)
    g = torch.randn(batch, rows, cols, generator=gen, device="cuda").to(getattr(torch, dtype))
    out = torch.full_like(g, float("nan"))
    ws = torch.full((readout.orthogonalize_workspace_bytes(batch, rows, cols),), 255, dtype=torch.uint8, device="cuda")
    for steps, coef in ((5, MUON), (0, MUON), (1, MUON), (8, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0))):
        readout.orthogonalize(g, out, ws, steps=steps, coefficients=coef)
        want = newton_schulz(torch, g, steps, coef, 1e-7, torch.float64)
        bound = orth_bound(g, newton_schulz(torch, g, steps, coef, 1e-7, torch.float32), want)
        if dtype == "bfloat16":
            bound += U16 * float(want.norm())
        assert float((out.double() - want).norm()) <= bound, (steps, coef)


def test_orthogonalize_reaches_orthogonality():
    """With coefficients that converge, the rows of the result are orthonormal: X X^T = 1 to a few roundings."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("orthonormal rows")
    g = torch.randn(1, 96, 300, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    ws = torch.empty(readout.orthogonalize_workspace_bytes(1, 96, 300), dtype=torch.uint8, device="cuda")
    readout.orthogonalize(g, g, ws, steps=16, coefficients=(1.875, -1.25, 0.375))
    x = g[0].double()
    assert float((x @ x.t() - torch.eye(96, device="cuda")).abs().max()) <= 32 * 2.0 ** -22


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_orthogonalize_strides_and_in_place(dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize strides {dtype}")
    gen = torch.Generator("cuda").manual_seed(8)
    for rows, cols in ((50, 77), (77, 50)):
        flat = torch.full((3, rows + 2, cols + 3), float("nan"), device="cuda").to(getattr(torch, dtype))
        g = flat[:, 1:rows + 1, 2:cols + 2]
        g.copy_(torch.randn(3, rows, cols, generator=gen, device="cuda"))
        nans = int(flat.isnan().sum())
        dense = g.contiguous()
        want = torch.empty_like(dense)
        ws = torch.empty(readout.orthogonalize_workspace_bytes(3, rows, cols), dtype=torch.uint8, device="cuda")
        readout.orthogonalize(dense, want, ws)
        readout.orthogonalize(g, g, ws)
        assert torch.equal(g, want) and int(flat.isnan().sum()) == nans
        one = torch.empty_like(dense[1])
        readout.orthogonalize(dense[1], one, ws)
        assert torch.equal(one, want[1])


@pytest.mark.parametrize("scale", [1e-30, 1e-9, 1e-4, 1e6, 1e25])
def test_orthogonalize_scales(scale):
    """Any size of update: the norm neither overflows nor vanishes; one far below eps only grows by a, step by step."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize scale {scale}")
    g = scale * torch.randn(1, 40, 90, generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    out = torch.empty_like(g)
    ws = torch.empty(readout.orthogonalize_workspace_bytes(1, 40, 90), dtype=torch.uint8, device="cuda")
    readout.orthogonalize(g, out, ws, eps=1e-7)
    want = newton_schulz(torch, g, 5, MUON, 1e-7, torch.float64)
    # from 2^-20 a product, at most fourfold a step
    assert float((out.double() - want).norm()) <= 2.0 ** -20 * 4 * float(want.norm())


def test_orthogonalize_zeros_and_not_finite():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("orthogonalize zeros, NaN")
    g = torch.randn(4, 20, 30, generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    g[0] = 0
    g[2, 3, 4] = float("nan")
    alone = torch.empty_like(g[1])
    out = torch.empty_like(g)
    ws = torch.empty(readout.orthogonalize_workspace_bytes(4, 20, 30), dtype=torch.uint8, device="cuda")
    readout.orthogonalize(g, out, ws)
    readout.orthogonalize(g[1], alone, ws)
    assert not out[0].any() and bool(out[2].isnan().all()) and torch.equal(out[1], alone) and bool(out[3].isfinite().all())


def test_orthogonalize_in_a_graph():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("orthogonalize graph")
    g = torch.randn(2, 100, 150, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    out = torch.empty_like(g)
    ws = torch.empty(readout.orthogonalize_workspace_bytes(2, 100, 150), dtype=torch.uint8, device="cuda")
    readout.orthogonalize(g, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        readout.orthogonalize(g, out, ws, stream=torch.cuda.current_stream())
    for k in range(4):
        g.add_(0.1 * k)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        readout.orthogonalize(g, out, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, got), f"replay {k}"


# ------------------------------------------------------------------------------------------------

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx_reference(x):
    """Codes and scale bytes of the rows of x (float64), by the definition."""
    rows, n = x.shape
    blocks = 4 * -(-n // 128)
    v = np.zeros((rows, blocks * 32))
    v[:, :n] = x
    v = v.reshape(rows, blocks, 32)
    top = np.abs(v).max(2)
    bad = ~np.isfinite(top)
    e = np.floor(np.log2(np.where(bad | (top == 0), 1.0, top))) - 2
    e = np.clip(np.where(top == 0, -127, e), -127, 127)
    s = np.where(bad[:, :, None], 0.0, np.abs(v)) / np.exp2(e)[:, :, None]
    far = np.abs(np.minimum(s, 6)[..., None] - GRID)
    even = np.arange(8) % 2  # a tie goes to the even code
    code = np.lexsort((np.broadcast_to(even, far.shape), far), axis=-1)[..., 0]
    code = code + 8 * (np.signbit(v) & ~bad[:, :, None])
    code = code.reshape(rows, -1).astype(np.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, np.where(bad, 255, e + 127).astype(np.uint8)


def mx_values(codes, scales):
    c = np.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1, 32)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0) * np.exp2(scales[:, :, None].astype(np.float64) - 127)
    return np.where(scales[:, :, None] == 255, np.nan, v).reshape(codes.shape[0], -1)


def quantized(torch, readout, x):
    nb = readout.mx_blocks(x.shape[1])
    codes = torch.full((x.shape[0], 16 * nb), 255, dtype=torch.uint8, device="cuda")
    scales = torch.full((x.shape[0], nb), 9, dtype=torch.uint8, device="cuda")
    readout.mx_quantize(x, codes, scales)
    return codes, scales


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n,pad,offset", [(1, 1, 0, 0), (2, 31, 0, 0), (3, 33, 2, 1), (4, 128, 0, 0), (5, 129, 8, 8), (64, 1000, 0, 0), (7, 4096, 0, 3), (1000, 65, 0, 0)])
def test_mx_quantize(rows, n, pad, offset, dtype):
    """Every code and scale byte, ties and each binary order of magnitude among the values; and the values they stand for."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"quantize {rows} x {n} {dtype}")
    gen = torch.Generator("cuda").manual_seed(n)
    dt = getattr(torch, dtype)
    x = matrix(torch, gen, rows, n, dt, 1.0, pad, offset)
    x[::2] = (x[::2] * 8).round() / 4  # ties
    x *= torch.exp2(torch.randint(-30, 30, (rows, 1), generator=gen, device="cuda").float()).to(dt)
    codes, scales = quantized(torch, readout, x)
    want = mx_reference(x.double().cpu().numpy())
    np.testing.assert_array_equal(scales.cpu().numpy(), want[1])
    np.testing.assert_array_equal(codes.cpu().numpy(), want[0])
    out = matrix(torch, gen, rows, n, dt, 1.0, pad, offset)
    readout.mx_dequantize(codes, scales, out)
    np.testing.assert_array_equal(out.double().cpu().numpy(), mx_values(*want)[:, :n])


def test_mx_special_values():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("quantize special values")
    x = torch.zeros(12, 64, device="cuda")
    x[0, 3] = float("nan")
    x[1, 40] = -float("inf")
    x[2, :2] = torch.tensor([3.4e38, -1.0], device="cuda")
    x[3, :2] = torch.tensor([2.0 ** -126, 2.0 ** -127], device="cuda")
    x[4, :3] = torch.tensor([2.0 ** -149, -2.0 ** -140, 2.0 ** -128], device="cuda")
    x[5] = -0.0
    x[6, :9] = torch.tensor([7.99, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0], device="cuda")
    x[7, :4] = torch.tensor([4.0, 0.2500001, 0.2499999, 6.5], device="cuda")
    x[8, 32:] = 1.0
    x[9, :3] = torch.tensor([2.0 ** -125, 3.0 * 2.0 ** -128, 2.0 ** -124], device="cuda")
    codes, scales = quantized(torch, readout, x)
    want = mx_reference(x.double().cpu().numpy())
    np.testing.assert_array_equal(scales.cpu().numpy(), want[1])
    np.testing.assert_array_equal(codes.cpu().numpy(), want[0])
    out = torch.empty_like(x)
    readout.mx_dequantize(codes, scales, out)
    np.testing.assert_array_equal(out.double().cpu().numpy(), mx_values(*want)[:, :64])


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 1000, 4096), (2, 33, 100), (15, 257, 129), (16, 64, 256), (17, 300, 1000), (40, 2000, 640), (64, 10, 3001), (130, 140, 384), (257, 1021, 511),
            (700, 3, 200), (4, 9000, 64), (33, 70, 16384)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,outputs,n", PRODUCTS)
def test_mx_product_and_linear(rows, outputs, n, dtype):
    """Products of two codes are exact: the sums' rounding is all, (n / 128 + 8) fp32 roundings, and the output's."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"mx product {rows} x {outputs} x {n} {dtype}")
    gen = torch.Generator("cuda").manual_seed(n)
    dt = getattr(torch, dtype)
    x = matrix(torch, gen, rows, n, dt, 2.0, n % 3, 0)
    w = torch.randn(outputs, n, generator=gen, device="cuda") * torch.exp2(torch.arange(outputs, device="cuda") % 7 - 3.0)[:, None]
    qx, qw = quantized(torch, readout, x), quantized(torch, readout, w)
    out = matrix(torch, gen, rows, outputs, dt, 1.0, rows % 3, 0)
    readout.mx_product(*qx, *qw, n, out)
    vx, vw = (torch.from_numpy(mx_values(*(t.cpu().numpy() for t in q))).cuda() for q in (qx, qw))
    want = vx @ vw.t()
    bound = (n / 128 + 8) * U32 * (vx.abs() @ vw.abs().t()) + (U16 if dtype == "bfloat16" else U32) * want.abs() * 1.01
    assert float(((out.double() - want).abs() - bound).max()) <= 0
    again = torch.full_like(out, float("nan"))
    ws = torch.full((readout.mx_linear_workspace_bytes(rows, n),), 255, dtype=torch.uint8, device="cuda")
    readout.mx_linear(x, *qw, again, ws)
    # the same sums, perhaps of more or fewer parts
    assert float(((again.double() - want).abs() - bound).max()) <= 0


def test_mx_product_of_nan_blocks():
    """A NaN block makes NaN of its row's (or column's) outputs and of nothing else."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("mx product NaN")
    for rows in (5, 100):
        x = torch.randn(rows, 300, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
        w = torch.randn(50, 300, generator=torch.Generator("cuda").manual_seed(2), device="cuda")
        x[3, 299], w[7, 0] = float("inf"), float("nan")
        out = torch.empty(rows, 50, device="cuda")
        ws = torch.empty(readout.mx_linear_workspace_bytes(rows, 300), dtype=torch.uint8, device="cuda")
        readout.mx_linear(x, *quantized(torch, readout, w), out, ws)
        nan = out.isnan()
        want = torch.zeros_like(nan)
        want[3], want[:, 7] = True, True
        assert torch.equal(nan, want)


def test_mx_linear_in_a_graph_and_on_a_stream():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("mx graph")
    gen = torch.Generator("cuda").manual_seed(1)
    qw = quantized(torch, readout, torch.randn(300, 512, generator=gen, device="cuda"))
    for rows in (1, 70):
        x = torch.randn(rows, 512, generator=gen, device="cuda")
        out, want = torch.empty(rows, 300, device="cuda"), torch.empty(rows, 300, device="cuda")
        ws = torch.empty(readout.mx_linear_workspace_bytes(rows, 512), dtype=torch.uint8, device="cuda")
        readout.mx_linear(x, *qw, out, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            readout.mx_linear(x, *qw, out, ws, stream=torch.cuda.current_stream())
        side = torch.cuda.Stream()
        for k in range(3):
            x.add_(1.0)
            graph.replay()
            torch.cuda.synchronize()
            readout.mx_linear(x, *qw, want, ws, stream=side)
            side.synchronize()
            assert torch.equal(out, want)


def test_binding_refuses_wrong_tensors():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("refusals")
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    y, v = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for bad in (dict(x=x.half()), dict(x=x.t()), dict(w=w[:, :7]), dict(w=w.bfloat16()), dict(labels=y.int()), dict(labels=y[:3]), dict(loss=v.double()), dict(lse=v[::2]),
                dict(x=x.cpu()), dict(workspace=ws.cpu()), dict(x=v)):
        with pytest.raises(ValueError):
            readout.loss(**{**dict(x=x, w=w, labels=y, loss=v, lse=v, workspace=ws), **bad})
    for bad in (dict(dx=x[:3]), dict(dw=w.bfloat16()), dict(row_grad=y), dict(lse=v.double())):
        with pytest.raises(ValueError):
            readout.gradient(**{**dict(x=x, w=w, labels=y, lse=v, dx=x.clone(), dw=w.clone(), workspace=ws), **bad})
    with pytest.raises(readout.SdnnError) as e:
        readout.loss(x, w, y, v, v, ws[:256])
    assert e.value.name == "SDNN_ERANGE"
    with pytest.raises(ValueError):
        readout.orthogonalize(x, x.bfloat16(), ws)
    with pytest.raises(ValueError):
        readout.orthogonalize(x, x[:2], ws)
    c, s = torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.zeros(4, 4, dtype=torch.uint8, device="cuda")
    for bad in (dict(codes=c[:3]), dict(scales=s[:, :2]), dict(codes=c.int()), dict(x=torch.zeros(4, 129, device="cuda"))):
        with pytest.raises(ValueError):
            readout.mx_quantize(**{**dict(x=x, codes=c, scales=s), **bad})
    with pytest.raises(ValueError):
        readout.mx_linear(x, c, s, torch.zeros(4, 5, device="cuda"), ws)


def test_example():
    """The example trains: its loss falls below a tenth, and 4-bit answers stay right on nearly every row."""
    torch_cuda()
    log("example")
    from examples import readout as example
    got = example.main()
    log(str(got))
    assert got["rows"] > 1000 and got["last loss"] < 0.1 * got["first loss"] and got["right"] > 0.95 and got["right in 4 bits"] > 0.9


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,classes,features", [(6, 1000, 200), (200, 70, 64), (300, 2000, 130), (5, 3, 40)])
def test_labelled_rows_of_infinities_and_nan(dtype, rows, classes, features):
    """Such a row's loss is NaN; the other rows' bits are what they are without it."""
    log(f"readout infinities {dtype} {rows} {classes} {features}")
    c = Case(rows, classes, features, dtype, seed=11)
    t = c.torch
    c.run()
    loss, lse = c.loss.clone(), c.lse.clone()
    c.x[0, 1], c.x[2, 0], c.x[4, features - 1] = float("inf"), -float("inf"), float("nan")
    c.run()
    bad = t.zeros(rows, dtype=t.bool, device="cuda")
    bad[[0, 2, 4]] = True
    assert t.equal(c.loss.isnan(), bad) and t.equal(c.loss[~bad], loss[~bad]) and t.equal(c.lse[~bad], lse[~bad])


# one to four rows or classes against more, or longer, rows than the streaming kernels take: both sides of each limit
@pytest.mark.parametrize("rows,classes,features,dtype", [
    (1, 8192, 33, "float32"), (1, 8193, 33, "float32"), (1, 8193, 511, "float32"), (1, 8193, 512, "float32"), (8193, 1, 100, "float32"),
    (4, 8193, 100, "float32"), (3, 8192, 100, "float32"), (2, 8193, 2047, "float32"), (2, 8193, 2048, "float32"), (8193, 4, 130, "float32"), (8193, 3, 2050, "float32"),
    (1, 8193, 2048, "bfloat16"), (1, 8193, 2049, "bfloat16"), (8193, 1, 70, "bfloat16"), (1, 1024, 4100, "bfloat16"), (1, 1025, 4100, "bfloat16"), (1025, 1, 4098, "bfloat16")])
def test_few_against_many(rows, classes, features, dtype):
    log(f"readout few against many {rows} x {classes} x {features} {dtype}")
    c = Case(rows, classes, features, dtype, seed=features)
    if rows > 4:
        c.y[::3] = -1
    c.run()
    c.check()
    g = c.torch.randn(rows, generator=c.torch.Generator("cuda").manual_seed(1), device="cuda")
    c.run(g)
    c.check(g)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,classes,features", [(2100, 2100, 1030), (600, 8200, 515), (300, 14000, 2050)])
def test_millions_of_logits_in_parts(rows, classes, features, dtype):
    """Blocks for half of the CUs: their features are split, if that pays; labels are left out here and there."""
    log(f"readout logits in parts {rows} x {classes} x {features} {dtype}")
    c = Case(rows, classes, features, dtype, seed=rows)
    c.y[::5] = -1
    c.run()
    c.check()
