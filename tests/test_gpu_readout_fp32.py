"""The readout's fp32 gradient where rows, classes, features or weights differ by many powers of two, at more than 192 rows
and classes (the form whose operands are held in parts), against 64 bits.

Bounds. u = 2^-24. The logits are products of operands in two fp16 parts under a power of two of each row: off by at most
d = (6 k / 32 + 40) u + 4 * 2^-22 of a logit's sum of magnitudes plus 2^-38 k of its two rows' largest magnitudes. A
softmax of logits off by up to d lies between those of l - d and l + d; lse rounds by 2 u (1 + |lse|) beyond that, and exp's
argument and result by (|l - lse| + 8) 2^-22. G is those probabilities less one at the label, rounded twice (the subtraction,
the weight). dx and dw are sums of G in three bf16 parts (exact; products below 2^-24 of a term are left out), so each
value's error goes by its own sum of magnitudes, without a common floor: (6 k / 32 + 40) u + 4 u of it, what G's error
makes of it, and two roundings of the result."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import Case

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = 2.0 ** -100  # what parts below the normal numbers lose


def sums(k):
    return (6 * k / 32 + 40) * U


def check(c, g, certain=()):
    """`certain`: rows whose answer is certain and right; their part of G is zero to the bit."""
    t = c.torch
    live = (c.y >= 0) & (c.y < c.w.shape[0])
    x, w = t.where(live[:, None], c.x.double(), 0.0), c.w.double()
    l, k = x @ w.t(), x.shape[1]
    d = (sums(k) + 4 * 2.0 ** -22) * (x.abs() @ w.abs().t()) + 2.0 ** -38 * k * x.abs().amax(1)[:, None] * w.abs().amax(1)
    lse = t.logsumexp(l, 1)
    e = t.maximum(t.logsumexp(l + d, 1) - lse, lse - t.logsumexp(l - d, 1)) + 2 * U * (1 + lse.abs())
    p = t.exp(l - lse[:, None])
    ep = t.exp(l - lse[:, None] + d + e[:, None] + ((l - lse[:, None]).abs() + 8) * 2.0 ** -22) - p
    G = p.scatter_add(1, c.y.clamp(0, w.shape[0] - 1)[:, None], -t.ones_like(p[:, :1]))
    weight = t.where(live, t.full_like(lse, 1.0 / max(1, int(live.sum()))) if g is None else g.double(), 0.0)[:, None]
    for r in certain:
        G[r] = ep[r] = 0
        assert not c.dx[r].any(), f"row {r} is certain"
    G, eG = G * weight, (ep + 2 * U * G.abs()) * weight.abs()
    for name, got, a, ea, b in (("dx", c.dx, G, eG, w.t().contiguous()), ("dw", c.dw, G.t().contiguous(), eG.t().contiguous(), x.t().contiguous())):
        want, size = a @ b.t(), a.abs() @ b.abs().t()
        bound = (sums(a.shape[1]) + 4 * U) * size + 1.01 * (ea @ b.abs().t()) + 4 * U * want.abs() + TINY * float(b.abs().max())
        assert bool(got.isfinite().all()), f"{name} is not finite"
        over = ((got.double() - want).abs() / bound).amax()
        assert float(over) <= 1.0, f"{name} is {float(over):.3g} times its bound off"


SIZES = [(200, 300, 64), (257, 1000, 129), (700, 201, 33)]


def weights(c, which):
    if which == "mean":
        return None
    gen = c.torch.Generator("cuda").manual_seed(7)
    return c.torch.randn(len(c.y), generator=gen, device="cuda") * c.torch.exp2(-(c.torch.arange(len(c.y), device="cuda") % 40.0))


@pytest.mark.parametrize("which", ["mean", "weights"])
@pytest.mark.parametrize("size", [1.0, 1e4, 1e8, 1e12, 1e20])
@pytest.mark.parametrize("rows,classes,features", SIZES)
def test_one_row_far_larger(rows, classes, features, size, which):
    """A labelled row `size` times the others, whose answer is certain and right: the others' gradients are theirs."""
    log(f"readout fp32 one row {size:g} times {rows} x {classes} x {features} {which}")
    c = Case(rows, classes, features, "float32", seed=3)
    certain = ()
    if size > 1:
        c.x[3] *= size
        l = c.x[3].double() @ c.w.double().t()
        c.y[3] = l.argmax()
        if size >= 1e8:  # (at 1e4 the next class may be near)
            certain = (3,)
    if size == 1e4:
        c.y[3] = -1
    g = weights(c, which)
    c.run(g)
    check(c, g, certain)


@pytest.mark.parametrize("which", ["mean", "weights"])
@pytest.mark.parametrize("size", [1e4, 1e8, 1e12, 1e20])
@pytest.mark.parametrize("rows,classes,features", SIZES)
def test_one_class_far_larger(rows, classes, features, size, which):
    """A class's weights `size` times the others' and negative against rows that are not: no row answers it."""
    log(f"readout fp32 one class {size:g} times {rows} x {classes} x {features} {which}")
    c = Case(rows, classes, features, "float32", seed=4)
    c.w[5] = -size * c.w[5].abs()
    c.y[c.y == 5] = 6
    g = weights(c, which)
    c.run(g)
    check(c, g)


@pytest.mark.parametrize("rows,classes,features", SIZES)
def test_features_of_many_sizes(rows, classes, features):
    """Features 30 binary orders apart: the gradient of the smallest is as good as that of the largest."""
    log(f"readout fp32 features {rows} x {classes} x {features}")
    c = Case(rows, classes, features, "float32", seed=5)
    c.x *= c.torch.exp2(-(c.torch.arange(features, device="cuda") % 31.0))
    c.run()
    check(c, None)


def test_values_at_the_ends_of_fp32():
    """Rows and weights near fp32's largest and smallest: nothing turns infinite on the way, the small ones count."""
    log("readout fp32 ends")
    c = Case(250, 240, 40, "float32", seed=6)
    c.x[2], c.x[4] = 3.4e38 * (c.x[2] > 0), 1e-30 * c.x[4]
    c.w *= 1e-38  # logits up to about 1
    c.w[7] = 1e-37
    c.run()
    assert bool(c.loss.isfinite().all()) and bool(c.dx.isfinite().all()) and bool(c.dw.isfinite().all())
    l = c.x.double() @ c.w.double().t()
    G = c.torch.softmax(l, 1)
    G[c.torch.arange(250), c.y] -= 1
    want = G.t() @ c.x.double() / 250
    size = (G.t().abs() @ c.x.double().abs()) / 250
    # (logits within 2^-20 of their magnitudes, at most 40 * 4 of them a row)
    assert float(((c.dw.double() - want).abs() - 160 * 2.0 ** -20 * size).max()) <= 0


def case(**kw):
    """Sizes on which both operands go in parts."""
    c = Case(**{**dict(rows=211, classes=300, features=97, dtype="float32", seed=9), **kw})
    assert min(c.x.shape[0], c.w.shape[0]) > 192
    return c


@pytest.mark.parametrize("pad,offset", [(0, 0), (0, 1), (1, 0), (8, 0), (3, 5), (24, 8)])
@pytest.mark.parametrize("features", [33, 64, 96, 97, 129])
def test_strides_and_alignment(features, pad, offset):
    """Rows apart from each other, bases on any value, NaN all around: nothing outside a matrix is used or written."""
    log(f"readout fp32 strides {features} {pad} {offset}")
    c = case(features=features, pad=pad, offset=offset)
    around = [t.as_strided((t.untyped_storage().nbytes() // t.element_size(),), (1,), 0) for t in (c.dx, c.dw)]
    before = [a.isnan().sum() for a in around]
    for which in ("mean", "weights"):
        g = weights(c, which)
        c.run(g)
        check(c, g)
    assert [a.isnan().sum() for a in around] == before


def test_rows_without_a_label():
    """They hold NaN, infinities and huge values, and so do their weights; labels are below, at and past the ends."""
    log("readout fp32 masked rows")
    c = case()
    t = c.torch
    out = t.tensor([0, 3, 64, 65, 100, 210], device="cuda")
    c.y[out] = t.tensor([-1, 300, -100, 1 << 40, -(1 << 62), 301], device="cuda")
    c.x[0], c.x[3, 5], c.x[64], c.x[65, 0], c.x[100] = float("nan"), float("inf"), -float("inf"), 3e38, 1e30
    g = t.rand(211, device="cuda")
    g[out] = float("nan")
    for w in (None, g):
        c.run(w)
        check(c, None if w is None else t.where(w.isnan(), 0.0, w))
        assert not c.loss[out].any() and not c.dx[out].any()


def test_no_row_has_a_label():
    log("readout fp32 all masked")
    c = case()
    c.y.fill_(-1)
    c.x.fill_(float("nan"))
    c.run()
    assert not c.loss.any() and not c.dx.any() and not c.dw.any()


@pytest.mark.parametrize("what", ["dx", "dw"])
def test_one_gradient_alone(what):
    log(f"readout fp32 {what} alone")
    c = case()
    c.run()
    want = getattr(c, what).clone()
    getattr(c, what).fill_(5)
    c.ws.fill_(255)
    c.r.gradient(c.x, c.w, c.y, c.lse, c.dx if what == "dx" else None, c.dw if what == "dw" else None, c.ws)
    assert c.torch.equal(getattr(c, what), want)


def test_labelled_rows_of_infinities_and_nan():
    """Such a row has a NaN in its loss and its dx, and makes NaN of dw; the other rows' dx are what they are without it."""
    log("readout fp32 infinities")
    c = case()
    c.run()
    dx, lse = c.dx.clone(), c.lse.clone()
    c.x[0, 1], c.x[2, 0], c.x[4, 96] = float("inf"), -float("inf"), float("nan")
    c.run()
    bad = c.torch.zeros(211, dtype=c.torch.bool, device="cuda")
    bad[[0, 2, 4]] = True
    assert c.torch.equal(c.dx.isnan().any(1), bad) and c.torch.equal(c.dx[~bad], dx[~bad]) and c.torch.equal(c.lse[~bad], lse[~bad])
    assert bool(c.loss[bad].isnan().all()) and bool(c.dw.isnan().any())


def test_gradient_against_differences():
    """Directional derivatives of the loss as the library computes it: the loss's error is at most 1e-5 a row, that of the
    quotient at h^2 / 6 times the third derivative, at most the cube of twice the logits' largest change along the direction."""
    log("readout fp32 differences")
    c = case(features=64)
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


def test_several_pieces():
    """More classes than a piece of G holds, the last one ragged; a row and a class far larger than the others."""
    log("readout fp32 pieces")
    c = Case(2100, 33000, 40, "float32", seed=15)
    c.y[::7] = -1
    c.x[3] *= 1e8
    c.y[3] = (c.x[3].double() @ c.w.double().t()).argmax()
    c.run()
    check(c, None, (3,))
