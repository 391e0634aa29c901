"""The gated hidden layer on the GPU against a plain evaluation in 64 bits.

Bounds. u16 = 2^-8 and u32 = 2^-24 are the unit roundoffs of bf16 and fp32. A sum of k products in fp32 is off by at most
s(k) = (k / 4 + 40) u32 times the sum of magnitudes: the matrix instructions take 4 products (fp32) or 32 (16-bit, at most
6 slabs of them for a group of fp32 products) into a sum at a time, and the parts of a split k, at most 64, meet in one more
chain, which 40 holds with the few roundings around it. fp32 inputs in two fp16 parts add 4 * 2^-22 times the magnitudes and
2^-38 k times the largest ones. From the sums' bounds eg and eu: act changes by at most 1.13 eg (the largest slope of
silu is 1.10, of gelu 1.13), its slope by at most 0.8 eg (silu 0.5, gelu 0.8; relu's is exact where g is), and either
is computed within (g^2 + |g| + 8) 2^-22 of its size (or of |g| + 1, for the slope): exp's and erfc's argument is rounded
once. Kept g and u, dg, du and the results are rounded to the tensors' type, once each."""
import math

import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import assert_within, matrix

pytestmark = pytest.mark.gpu
U16, U32 = 2.0 ** -8, 2.0 ** -24


def sum_bound(k):
    return (k / 4 + 40) * U32


def product_bound(a, b, fp32):
    """Elementwise bound of the error of a b^T (rows of a, rows of b)."""
    k = a.shape[1]
    e = (sum_bound(k) + (4 * 2.0 ** -22 if fp32 else 0)) * (a.abs() @ b.abs().t())
    return e + 2.0 ** -38 * k * a.abs().max() * b.abs().max() if fp32 else e


def activation(torch, name, g):
    """act(g) and its slope."""
    if name == "relu":
        return g.clamp(min=0), (g > 0).double()
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1 - p)
    p = torch.special.ndtr(g)
    return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def reference(torch, act, x, wg, wu, dh):
    """(value, bound) of g, u, h, dx, dwg, dwu."""
    fp32 = x.dtype == torch.float32
    unit = U32 if fp32 else U16
    x, wg, wu, dh = (v.double() for v in (x, wg, wu, dh))
    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = product_bound(x, wg, fp32), product_bound(x, wu, fp32)
    a, slope = activation(torch, act, g)
    step = (g * g + g.abs() + 8) * 2.0 ** -22
    ea = 1.13 * eg + step * a.abs()
    h = a * u
    eh = ea * (u.abs() + eu) + a.abs() * eu + 2 * U32 * h.abs()
    # the gradient has g and u as they are kept
    kg, ku = eg + unit * (g.abs() + eg), eu + unit * (u.abs() + eu)
    ka = 1.13 * kg + step * a.abs()
    es = (0.0 if act == "relu" else 0.8) * kg + step * (g.abs() + 1)
    dg, du = dh * u * slope, dh * a
    edg = dh.abs() * (es * (u.abs() + ku) + slope.abs() * ku) + 3 * U32 * dg.abs()
    edu = dh.abs() * ka + 2 * U32 * du.abs()
    edg, edu = (e + (2.0 ** -22 if fp32 else U16) * (d.abs() + e) for e, d in ((edg, dg), (edu, du)))

    def product(d, ed, m):  # d m with rows of k in m
        return d @ m, ed @ m.abs() + product_bound(d.abs() + ed, m.t().contiguous(), False) + (4 * 2.0 ** -22 if fp32 else 0) * (d.abs() @ m.abs())

    (x1, e1), (x2, e2) = product(dg, edg, wg), product(du, edu, wu)
    extra = sum_bound(2 * g.shape[1]) * (dg.abs() @ wg.abs() + du.abs() @ wu.abs())  # one sum goes through both
    out = [(g, eg), (u, eu), (h, eh), (x1 + x2, e1 + e2 + extra), product(dg.t(), edg.t(), x), product(du.t(), edu.t(), x)]
    return [(v, e + unit * (v.abs() + e)) for v, e in out]


class Case:
    def __init__(self, rows, hidden, features, dtype, act="silu", seed=0, pad=0, offset=0, whole=False):
        from paper_1909_05631_amd import readout
        self.torch = torch = torch_cuda()
        self.r, self.act = readout, act
        gen = torch.Generator("cuda").manual_seed(seed)
        dt = getattr(torch, dtype)
        make = lambda *s, scale=1.0: matrix(torch, gen, *s, dt, scale, pad, offset)  # noqa: E731
        self.x = make(rows, features)
        self.wg, self.wu = (make(hidden, features, scale=1.5 / math.sqrt(features)) for _ in range(2))
        if whole:  # sums exact in fp32, zeros among them
            for t in (self.x, self.wg, self.wu):
                t.copy_(torch.randint(-1, 2, t.shape, generator=gen, device="cuda"))
        self.dh = make(rows, hidden, scale=0.1)
        self.h, self.gate, self.up = (make(rows, hidden).fill_(7) for _ in range(3))
        self.dx, self.dwg, self.dwu = (make(*t.shape).fill_(7) for t in (self.x, self.wg, self.wu))
        self.ws = torch.full((max(1, readout.gated_workspace_bytes(rows, hidden, features, dt, kept=False)),), 255, dtype=torch.uint8, device="cuda")

    def run(self, kept=True, stream=None):
        keep = dict(gate=self.gate, up=self.up) if kept else {}
        self.r.gated(self.x, self.wg, self.wu, self.h, self.ws, activation=self.act, stream=stream, **keep)
        self.r.gated_gradient(self.x, self.wg, self.wu, self.dh, self.dx, self.dwg, self.dwu, self.ws, activation=self.act, stream=stream, **keep)

    def outputs(self):
        return {"h": self.h, "dx": self.dx, "dwg": self.dwg, "dwu": self.dwu}

    def check(self, kept=True):
        want = dict(zip(("gate", "up", "h", "dx", "dwg", "dwu"), reference(self.torch, self.act, self.x, self.wg, self.wu, self.dh)))
        for name, got in ([("gate", self.gate), ("up", self.up)] if kept else []) + list(self.outputs().items()):
            assert_within(name, got, want[name])


SHAPES = [(1, 1, 1), (1, 16, 64), (1, 300, 1000), (2, 17, 3), (3, 1000, 130), (4, 33, 31), (5, 100, 257), (16, 129, 65), (17, 64, 128), (33, 31, 40), (64, 256, 128), (100, 10, 1024), (200, 193, 72),
          (257, 1000, 72), (300, 2047, 40), (1021, 130, 500), (700, 700, 260), (2500, 300, 33), (3, 9000, 64), (1, 40, 9000), (300, 20, 5000), (192, 500, 65), (193, 500, 65), (300, 500, 65), (301, 500, 65),
          (500, 192, 65), (500, 301, 65), (700, 300, 65)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,hidden,features", SHAPES)
def test_layer_and_gradient(rows, hidden, features, dtype):
    log(f"gated {rows} x {hidden} x {features} {dtype}")
    c = Case(rows, hidden, features, dtype, act=("silu", "gelu")[(rows + hidden) % 2], seed=rows)
    c.run()
    c.check()
    kept = {k: v.clone() for k, v in c.outputs().items()}
    for v in c.outputs().values():
        v.fill_(3)
    c.run(kept=False)
    for k, v in c.outputs().items():
        assert c.torch.equal(v, kept[k]), f"{k} differs where g and u are computed again"


@pytest.mark.parametrize("rows,hidden,features,pad,offset", [(310, 2048, 1000, 0, 0), (1021, 2047, 1000, 0, 0), (2049, 640, 262, 3, 5), (1100, 402, 1501, 1, 0), (1055, 417, 1503, 0, 1),
                                                              (8192, 400, 400, 24, 8), (400, 4000, 1030, 0, 0), (193, 2048, 1000, 0, 0), (1000, 200, 1400, 0, 2), (2500, 97, 1200, 0, 0)])
def test_gradient_of_middle_sizes(rows, hidden, features, pad, offset):
    """fp32: about a block of 128 x 128 outputs for every CU; rows, outputs and features that end inside one, and inside a step
    of 32; split sums, and one of the results alone."""
    log(f"gated {rows} x {hidden} x {features} {pad} {offset}")
    c = Case(rows, hidden, features, "float32", act="gelu", seed=hidden, pad=pad, offset=offset)
    around = [t.as_strided((t.untyped_storage().nbytes() // t.element_size(),), (1,), 0) for t in (c.dx, c.dwg, c.dwu)]
    before = [a.isnan().sum() for a in around]
    c.run()
    c.check()
    assert [a.isnan().sum() for a in around] == before
    kept = {k: v.clone() for k, v in c.outputs().items()}
    for only in ("dx", "dwg", "dwu"):
        v = c.outputs()[only]
        v.fill_(3)
        to = [v if name == only else None for name in ("dx", "dwg", "dwu")]
        c.r.gated_gradient(c.x, c.wg, c.wu, c.dh, *to, c.ws, activation=c.act, gate=c.gate, up=c.up)
        assert c.torch.equal(v, kept[only]), only


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_activations_of_exact_sums(act, dtype):
    """Whole numbers: g is exact, zero among its values, where relu's slope is 0."""
    log(f"gated {act} {dtype}")
    for rows, hidden in ((70, 90), (300, 400)):
        c = Case(rows, hidden, 50, dtype, act=act, seed=2, whole=True)
        c.run()
        c.check()
        assert bool((c.gate == 0).any())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (8, 0), (3, 5), (24, 8)])
def test_strides_and_alignment(pad, offset, dtype):
    """Rows apart from each other, bases on any value, NaN all around: nothing outside a matrix is used or written."""
    log(f"gated strides {pad} {offset} {dtype}")
    for rows, hidden, features in ((70, 140, 96), (3, 141, 97), (210, 205, 98)):
        c = Case(rows, hidden, features, dtype, seed=3, pad=pad, offset=offset)
        around = [t.as_strided((t.untyped_storage().nbytes() // t.element_size(),), (1,), 0) for t in (c.dx, c.dwg, c.dwu, c.h, c.gate, c.up)]
        before = [a.isnan().sum() for a in around]
        c.run()
        c.check()
        assert [a.isnan().sum() for a in around] == before


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_matrices_of_different_strides(dtype):
    """One weight in place, one that has to be copied, x transposed into rows that are far apart."""
    log(f"gated mixed strides {dtype}")
    torch = torch_cuda()
    c = Case(40, 70, 66, dtype, seed=4)
    wide = torch.full((70, 71), float("nan"), dtype=c.wu.dtype, device="cuda")
    wide[:, 5:] = c.wu
    c.wu = wide[:, 5:]
    far = torch.full((40, 300), float("nan"), dtype=c.x.dtype, device="cuda")
    far[:, 10:76] = c.x
    c.x = far[:, 10:76]
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("what", ["dx", "dwg", "dwu"])
def test_one_gradient_alone(what, dtype):
    log(f"gated {what} alone {dtype}")
    for rows in (90, 400):
        c = Case(rows, 300, 64, dtype)
        c.run()
        want = {k: v.clone() for k, v in c.outputs().items()}
        for k in ("dx", "dwg", "dwu"):
            getattr(c, k).fill_(5)
        args = [getattr(c, k) if k == what else None for k in ("dx", "dwg", "dwu")]
        c.r.gated_gradient(c.x, c.wg, c.wu, c.dh, *args, c.ws, activation=c.act, gate=c.gate, up=c.up)
        for k in ("dx", "dwg", "dwu"):
            assert c.torch.equal(getattr(c, k), want[k]) if k == what else bool((getattr(c, k) == 5).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_rows(dtype):
    log(f"gated no rows {dtype}")
    c = Case(0, 9, 40, dtype)
    c.run()
    assert not c.dwg.any() and not c.dwu.any()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_infinities_and_nan_stay_in_their_rows(dtype):
    """A row that is not finite reaches its own h and dx and, through dg and du, the weights' gradients; other rows' h and
    dx are those of a batch without it."""
    log(f"gated not finite {dtype}")
    for rows in (5, 300):
        c = Case(rows, 210, 64, dtype, seed=8)
        t = c.torch
        c.run()
        good = c.h.clone(), c.dx.clone()
        c.x[1, 3], c.x[2, 0] = float("nan"), float("inf")
        c.run()
        rest = [i for i in range(rows) if i not in (1, 2)]
        assert bool(c.h[1].isnan().all()) and not bool(c.h[2].isfinite().all())
        assert t.equal(c.h[rest], good[0][rest]) and t.equal(c.dx[rest], good[1][rest])
        assert bool(c.dwg[:, 3].isnan().all())


def test_large_and_small_gates():
    """Values of g far out on either side: act and its slope have their limits, and nothing overflows on the way."""
    torch = torch_cuda()
    log("gated far values")
    for act in ("silu", "gelu"):
        c = Case(40, 16, 1, "float32", act=act)
        c.x.copy_(torch.tensor([-1e30, -1e4, -200.0, -104.0, -90.0, -88.0, -40.0, -13.0, -12.0, -5.0] * 2 + [1e30, 1e4, 200.0, 90.0, 88.0, 40.0, 17.0, 9.0, 5.0, 0.0] * 2).cuda()[:, None])
        c.wg.fill_(1.0)
        c.wu.fill_(2.0 ** -100)
        c.run()
        g = c.x.double()[:, :1].expand(-1, 16)
        a, slope = activation(torch, act, g)
        u = g * 2.0 ** -100
        # denormal results and those of an exponential that left the normal range are absolute errors of fp32's smallest
        assert_within("h", c.h, (a * u, (g.square().clamp(max=1e4) + g.abs().clamp(max=1e4) + 10) * 2.0 ** -22 * (a * u).abs() + 2.0 ** -126 * (1 + u.abs())))
        assert bool(c.dx.isfinite().all())


def test_rows_of_very_different_size():
    """fp32: a row or an output far larger than the others leaves these their precision."""
    log("gated wide range")
    for rows, hidden in ((40, 50), (300, 300), (310, 305)):
        c = Case(rows, hidden, 96, "float32", seed=9)
        c.x[7] *= 2.0 ** 40
        c.wu[11] *= 2.0 ** 30
        c.dh[13] *= 2.0 ** 30
        c.run()
        small = [i for i in range(rows) if i not in (7, 13)]
        out = [j for j in range(hidden) if j != 11]
        want = reference(c.torch, c.act, c.x[small], c.wg[out], c.wu[out], c.dh[small][:, out])
        for got, w in ((c.h[small][:, out], want[2]),):
            assert_within("h", got, w)
        # the weights' gradients without the large row's part, which is taken away in 64 bits: what is left of the others is
        # exact against the large row's rounding
        full = reference(c.torch, c.act, c.x, c.wg, c.wu, c.dh)
        for name, got, w in (("dwg", c.dwg[out], full[4]), ("dwu", c.dwu[out], full[5])):
            assert_within(name, got, (w[0][out], w[1][out]))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_against_differences(act):
    """Directional derivatives of sum(h * dh): (L(+e) - L(-e)) / 2e. Each h is within 2^-20 of its size and 1 (fp32, 64
    features of |x w| below 1), so that the quotient is off by at most sum |dh| (|h| + 1) 2^-20 / e, and by e^2 / 6 of a third
    derivative: with |g'|, |u'| <= r along the direction it is at most 3 r^3 (1 + |u|) a value."""
    log(f"gated differences {act}")
    c = Case(40, 30, 64, "float32", act=act, seed=11)
    t = c.torch
    c.run()
    e = 0.02
    gen = t.Generator("cuda").manual_seed(4)
    for name, grad in (("x", c.dx), ("wg", c.dwg), ("wu", c.dwu)):
        base = getattr(c, name).clone()
        d = t.randn(base.shape, generator=gen, device="cuda")
        d /= d.norm(dim=1, keepdim=True)
        total = []
        for sign in (1, -1):
            getattr(c, name).copy_(base + sign * e * d)
            c.r.gated(c.x, c.wg, c.wu, c.h, c.ws, activation=act)
            total.append(float((c.h.double() * c.dh.double()).sum()))
        getattr(c, name).copy_(base)
        r = (d.double() @ t.cat([c.wg, c.wu]).double().t() if name == "x" else c.x.double() @ d.double().t()).abs().max()
        want = float((grad.double() * d.double()).sum())
        size = float((c.dh.double().abs() * (c.h.double().abs() + 1)).sum())
        third = float((c.dh.double().abs() * (1 + c.up.double().abs())).sum()) * 3 * float(r) ** 3
        assert abs((total[0] - total[1]) / (2 * e) - want) <= size * 2.0 ** -20 / e + e * e / 6 * third


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_same_bits_on_any_stream_and_in_a_graph(dtype, rows):
    log(f"gated streams and graph {dtype} {rows}")
    c = Case(rows, 700, 200, dtype, seed=6)
    t = c.torch
    c.run()
    want = {k: v.clone() for k, v in c.outputs().items()}
    side = t.cuda.Stream()
    busy = t.rand(4096, 4096, device="cuda")
    t.cuda.synchronize()
    for v in c.outputs().values():
        v.fill_(3)
    side.wait_stream(t.cuda.current_stream())
    for _ in range(4):
        busy = busy @ busy * 1e-4
    c.run(stream=side)
    side.synchronize()
    assert all(t.equal(v, want[k]) for k, v in c.outputs().items())
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        c.run(kept=False, stream=t.cuda.current_stream())
    for k in range(4):
        c.x.mul_(0.5 + 0.25 * k)
        graph.replay()
        t.cuda.synchronize()
        got = {n: v.clone() for n, v in c.outputs().items()}
        for v in c.outputs().values():
            v.fill_(3)
        c.run(stream=t.cuda.current_stream())
        t.cuda.synchronize()
        assert all(t.equal(v, got[n]) for n, v in c.outputs().items()), f"replay {k}"


def test_binding_refuses():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("gated refusals")
    x, w, h = torch.zeros(4, 8, device="cuda"), torch.zeros(3, 8, device="cuda"), torch.zeros(4, 3, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for bad in (dict(x=x.half()), dict(x=x.t()), dict(w_gate=w[:, :7]), dict(w_up=w[:2]), dict(w_up=w.bfloat16()), dict(h=h[:3]), dict(h=h.double()), dict(gate=h[:, :2]), dict(up=h.bfloat16()),
                dict(x=x.cpu()), dict(workspace=ws.cpu()), dict(x=x[0]), dict(activation="tanh"), dict(activation=0), dict(activation=["silu"])):
        with pytest.raises(ValueError):
            readout.gated(**{**dict(x=x, w_gate=w, w_up=w.clone(), h=h, workspace=ws), **bad})
    for bad in (dict(dh=h[:3]), dict(dx=x[:3]), dict(dw_gate=w.bfloat16()), dict(dw_up=w[:, :3]), dict(gate=h[:2], up=h)):
        with pytest.raises(ValueError):
            readout.gated_gradient(**{**dict(x=x, w_gate=w, w_up=w.clone(), dh=h, dx=x.clone(), dw_gate=w.clone(), dw_up=w.clone(), workspace=ws), **bad})
    for call in (lambda: readout.gated(x, w, w.clone(), h, ws[:256]), lambda: readout.gated_gradient(x, w, w.clone(), h, x.clone(), None, None, ws[:256])):
        with pytest.raises(readout.SdnnError) as e:
            call()
        assert e.value.name == "SDNN_ERANGE"
    with pytest.raises(readout.SdnnError) as e:
        readout.gated_gradient(x, w, w.clone(), h, x.clone(), None, None, ws, gate=h.clone())
    assert e.value.name == "SDNN_EINVAL"
