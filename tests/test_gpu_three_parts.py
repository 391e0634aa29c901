"""fp32 operands in three bf16 parts, on sums of one product each: every part of both factors shows in the result.

Bounds. A value is its three parts exactly. Of the nine products of two values' parts six are taken; the others are at most
2^-26 of the value's product. The six meet in fp32, whatever their order, in at most six sums off by 2^-23 (the matrix
instructions may cut) of the largest partial sum, the value's own size: together 2^-20.4. The gradient's dg and du round once before, by
2^-24: 2^-20 in all. Without the third parts it is 2^-18 for either factor's.

Few rows of 4-bit weights: x's parts times -8 add up exactly (24 bits); their products with a code, at most three sums of at
most 8 |x|, or q |x| with offsets of zero; then one product and two sums with the scale."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import assert_within

PRODUCT = 2.0 ** -20


def full(torch, gen, *shape, device="cuda"):
    """Values of 24 bits in [1, 2) times 2^-3 to 2^3, of both signs."""
    bits = torch.randint(0, 1 << 23, shape, generator=gen, device=device).double() * 2.0 ** -23 + 1.0
    size = torch.randint(-3, 4, shape, generator=gen, device=device).double()
    sign = torch.randint(0, 2, shape, generator=gen, device=device) * 2.0 - 1.0
    return (sign * bits * 2.0 ** size).float()


def two_parts(torch, v):
    hi = v.bfloat16().float()
    return hi.double() + (v - hi).bfloat16().double()


def test_the_bounds_show_a_lost_part():
    """Products without the third part of one factor, exact otherwise: past the bound somewhere in any hundred of them."""
    import torch
    gen = torch.Generator().manual_seed(1)
    a, b = (full(torch, gen, 50, 100, device="cpu") for _ in range(2))
    value = a.double() * b.double()
    for lost in (two_parts(torch, a) * b, a * two_parts(torch, b), two_parts(torch, a) * two_parts(torch, b)):
        assert bool(((lost - value).abs() > PRODUCT * value.abs()).any(1).all())
    q = torch.randint(0, 16, a.shape, generator=gen).double()
    lost = (two_parts(torch, a) - a).abs()
    assert bool((lost * (q - 8).abs() > (24 * a.abs() + (q - 8).abs() * a.abs()) * 2.0 ** -23).any(1).all())
    assert bool((lost * q > 5 * q * a.abs() * 2.0 ** -23).any(1).all())


# Both kinds of blocks, whole and split sums, ends inside a block and inside a step of k.
SHAPES = [(301, 310, 70), (310, 305, 96), (500, 301, 65), (301, 500, 65), (1021, 2047, 1000), (600, 600, 600), (320, 330, 2000), (2049, 640, 262), (8192, 400, 400), (1055, 417, 1503)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,hidden,features", SHAPES)
def test_gradients_of_one_product(rows, hidden, features):
    """relu of positive gates: dg = dh u and du = dh g. Every column of x has one value, and every column of the two weights
    has one in one of them: each place of k in turn."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"gated gradient of one product {rows} x {hidden} x {features}")
    gen = torch.Generator("cuda").manual_seed(rows)
    gate, up, dh = full(torch, gen, rows, hidden).abs(), full(torch, gen, rows, hidden), full(torch, gen, rows, hidden)
    dg, du = dh.double() * up.double(), dh.double() * gate.double()
    both = torch.cat([dg, du], 1)
    x, dx = torch.zeros(rows, features, device="cuda"), torch.empty(rows, features, device="cuda")
    w = torch.zeros(2 * hidden, features, device="cuda")
    dwg, dwu = (torch.empty(hidden, features, device="cuda") for _ in range(2))
    ws = torch.full((readout.gated_workspace_bytes(rows, hidden, features, x.dtype),), 255, dtype=torch.uint8, device="cuda")
    column = torch.arange(features, device="cuda")
    for first in range(0, max(rows, 2 * hidden), features):
        t, j = (first + column) % rows, (first + column) % (2 * hidden)
        vx, vw = full(torch, gen, features), full(torch, gen, features)
        x.zero_()[t, column] = vx
        w.zero_()[j, column] = vw
        readout.gated_gradient(x, w[:hidden], w[hidden:], dh, dx, dwg, dwu, ws, activation="relu", gate=gate, up=up)
        for name, got, want in (("dx", dx, both[:, j] * vw.double()), ("dwg", dwg, dg[t].t() * vx.double()), ("dwu", dwu, du[t].t() * vx.double())):
            assert_within(f"{name} from {first}", got, (want, PRODUCT * want.abs()))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,outputs,n", [(1, 10, 31), (3, 300, 1000), (16, 129, 4096), (17, 40, 300), (33, 100, 1024), (64, 257, 520), (64, 130, 16384), (1, 40, 20001), (7, 50, 40000), (100, 4100, 4100),
                                            (256, 4096, 4096)])
def test_few_rows_of_one_product(rows, outputs, n):
    """Each row of x has one value, at places all over k and at its ends."""
    from paper_1909_05631_amd import readout
    from tests.test_gpu_grouped import Weights, parts_of
    torch = torch_cuda()
    log(f"grouped of one product {rows} x {n} to {outputs}")
    gen = torch.Generator("cuda").manual_seed(n)
    ends = torch.tensor([0, 1, 31, 32, 63, 64, 127, 128, n // 2, n - 33, n - 2, n - 1], device="cuda").clamp(0, n - 1)
    row = torch.arange(rows, device="cuda")
    x, out = torch.zeros(rows, n, device="cuda"), torch.empty(rows, outputs, device="cuda")
    ws = torch.full((max(1, readout.grouped_linear_workspace_bytes(rows, outputs, n, x.dtype)),), 255, dtype=torch.uint8, device="cuda")
    for group in readout.GROUPS:
        for offsets in (False, True):
            w = Weights(outputs, n, group, offsets, "float32", seed=group)
            if offsets:
                w.offsets.zero_()
            q, s, o = parts_of(w.codes, w.scales, w.offsets, n, group)
            for turn in range(max(1, 24 // rows)):
                k = torch.where((row + turn) % 2 == 0, ends[(row // 2 + turn * rows) % 12], torch.randint(0, n, (rows,), generator=gen, device="cuda"))
                v = full(torch, gen, rows)
                x.zero_()[row, k] = v
                readout.grouped_linear(x, w.codes, w.scales, out, ws, group=group, offsets=w.offsets)
                v, qk, sk = v.double()[:, None], q[:, k].t(), s[:, k].t()
                want = v * (qk * sk + o[:, k].t())
                assert_within("out", out, (want, 2.0 ** -23 * (5 * want.abs() if offsets else 24 * sk * v.abs() + want.abs())))
