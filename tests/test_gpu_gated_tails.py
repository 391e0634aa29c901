"""The activations' relative precision in fp32, far out on the side where they go to zero, on the GPU against 64 bits.

One row of one value 1, so that g and u are the weights to the bit and every result is one value's. Bounds, in units of
2^-24. silu: exp2 2 (its argument's rounding is taken back), the product with what was taken back 1, 1 + exp 1, the
reciprocal 2, two products 2: 8, and 16 are allowed. gelu's tail exp(-g^2 / 2) t p(t): exp2 and its correction 3; t, 3 for
the reciprocal and its argument, counts up to 2.5 times in t p(t); the polynomial's coefficients add up to 2.6 times its
value with two roundings each, and it is fitted to 2e-8: 6; three products and the value's two 5: 22, and 32 are allowed. A slope
is a sum whose terms have these errors."""
import math

import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import assert_within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,end,units", [("silu", 86.0, 16), ("gelu", 12.5, 32)])
def test_tails_keep_their_relative_precision(act, end, units):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"gated tail {act}")
    n = 40000
    g = -torch.linspace(1e-3, end, n, device="cuda", dtype=torch.float64).float()
    x = torch.ones(1, 1, device="cuda")
    wg, wu = g[:, None].contiguous(), torch.full((n, 1), 1.5 * 2.0 ** 60, device="cuda")  # (results stay far from fp32's smallest)
    h, dwg, dwu = torch.empty(1, n, device="cuda"), torch.empty_like(wg), torch.empty_like(wu)
    dh = torch.full((1, n), 2.0 ** 60, device="cuda")
    ws = torch.empty(readout.gated_workspace_bytes(1, n, 1, x.dtype, kept=False), dtype=torch.uint8, device="cuda")
    readout.gated(x, wg, wu, h, ws, activation=act)
    readout.gated_gradient(x, wg, wu, dh, None, dwg, dwu, ws, activation=act)
    g = g.double()
    if act == "silu":
        p = torch.sigmoid(g)
        value, terms = g * p, (p, g * p * (1 - p))
    else:
        p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        value, terms = g * p, (p, g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi))
    bound = units * 2.0 ** -24
    for name, got, size, parts in (("h", h[0], float(wu[0]), (value,)), ("dwu", dwu[:, 0], 2.0 ** 60, (value,)), ("dwg", dwg[:, 0], 2.0 ** 60 * float(wu[0]), terms)):
        assert_within(name, got, (size * sum(parts), bound * size * sum(t.abs() for t in parts)))
