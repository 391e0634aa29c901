"""The layer, the clipped gradients and the 4-bit weights at the ends of their sizes: the most outputs and features, a million
rows, results and lists past 2^31 values."""
import math

import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_gated import Case
from tests.test_gpu_gated import reference as layer_reference
from tests.test_gpu_grouped import Weights
from tests.test_gpu_grouped import reference as grouped_reference
from tests.test_gpu_readout import assert_within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,hidden,features", [(3, 1 << 19, 8), (20, 1 << 19, 8), (1 << 20, 8, 8), (5, 8, 1 << 20), (200, 200, 2500), (5000, 193, 40), (16, 24, 4096), (16, 24, 4100), (16, 40, 2100)])
def test_layer_and_gradient(rows, hidden, features, dtype):
    """Most of one size, few of the others; x that just fits a workgroup's LDS and x that does not."""
    log(f"gated ends {rows} x {hidden} x {features} {dtype}")
    c = Case(rows, hidden, features, dtype, seed=rows % 1000)
    c.run()
    c.check()


@pytest.mark.parametrize("rows,hidden", [(70000, 32768)])
def test_layer_of_more_than_two_to_the_31_results(rows, hidden):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("gated large")
    gen = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(rows, 32, generator=gen, device="cuda").bfloat16()
    wg, wu = (torch.randn(hidden, 32, generator=gen, device="cuda").div(6).bfloat16() for _ in range(2))
    h = torch.full((rows, hidden), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(readout.gated_workspace_bytes(rows, hidden, 32, x.dtype, gradient=False), dtype=torch.uint8, device="cuda")
    readout.gated(x, wg, wu, h, ws)
    at = torch.tensor([0, 255, 256, 32767, 65535, 65536, 65537, rows - 1], device="cuda")
    want = layer_reference(torch, "silu", x[at], wg, wu, torch.zeros(len(at), hidden, dtype=x.dtype, device="cuda"))[2]
    assert_within("h", h[at], want)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,outputs,n", [(1, 10, 1 << 20), (20, 10, 1 << 20), (1, 1 << 20, 32), (16, 16, 4352), (16, 16, 4353), (16, 16, 1152), (16, 16, 1153), (70, 17, 1 << 17)])
def test_linear(rows, outputs, n, dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"grouped ends {rows} x {n} to {outputs} {dtype}")
    dt = getattr(torch, dtype)
    w = Weights(outputs, n, 64, True, dtype)
    x = torch.randn(rows, n, device="cuda").to(dt)
    out = torch.full((rows, outputs), 7.0, dtype=dt, device="cuda")
    ws = torch.empty(max(1, readout.grouped_linear_workspace_bytes(rows, outputs, n, dt)), dtype=torch.uint8, device="cuda")
    readout.grouped_linear(x, w.codes, w.scales, out, ws, group=64, offsets=w.offsets)
    assert_within("out", out, grouped_reference(x, w.codes, w.scales, w.offsets, 64))


def test_linear_of_more_than_two_to_the_31_results():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("grouped large")
    rows, outputs = 70000, 32768
    w = Weights(outputs, 32, 32, False, "bfloat16")
    x = torch.randn(rows, 32, device="cuda").bfloat16()
    out = torch.full((rows, outputs), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(readout.grouped_linear_workspace_bytes(rows, outputs, 32, x.dtype), dtype=torch.uint8, device="cuda")
    readout.grouped_linear(x, w.codes, w.scales, out, ws, group=32)
    at = torch.tensor([0, 255, 256, 32767, 65535, 65536, 65537, rows - 1], device="cuda")
    # the bound of many rows, of which these are some (65 repeats of them, so that it is taken as many)
    many = at.repeat(9)
    value, bound = grouped_reference(x[many], w.codes, w.scales, w.offsets, 32)
    assert_within("out", out[at], (value[:8], bound[:8]))


def test_list_of_more_than_two_to_the_31_values():
    """One tensor past 2^31 values: its norm is known, and every value of the result."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("clip large")
    n = (1 << 31) + 9
    t = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    ws, norm = torch.empty(readout.clip_workspace_bytes(1), dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
    readout.clip([t], 1.0, norm, ws)
    want = math.sqrt(n) * 2.0 ** -10
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    value = 2.0 ** -10 / want
    assert float(t.min()) == float(t.max()) and abs(float(t[-1]) - value) <= (2.0 ** -8 + 3 * 2.0 ** -24) * value
