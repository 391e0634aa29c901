"""4-bit products of few rows: both sides of the rule between the kernel that streams the weights past a few rows and the
tiles, against 64 bits of the values that the codes stand for (exact products, (n / 128 + 8) fp32 roundings of the sums)."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import U16, U32, quantized

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,outputs,n", [(1, 70, 65536), (1, 70, 65537), (2, 100, 32768), (2, 100, 32769), (3, 9000, 700), (4, 9000, 1024), (5, 9000, 1024), (5, 9000, 768), (4, 50, 16384),
                                            (5, 50, 16384), (8, 8192, 4096), (8, 8193, 4096), (9, 100, 4096), (16, 8192, 2048), (16, 8193, 2048), (16, 8193, 256), (16, 30, 257), (17, 30, 100)])
def test_few_rows_and_the_tiles(rows, outputs, n, dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"mx few {rows} x {outputs} x {n} {dtype}")
    gen = torch.Generator("cuda").manual_seed(n + rows)
    x = (torch.randn(rows, n, generator=gen, device="cuda") * torch.exp2(torch.arange(rows, device="cuda") % 5 - 2.0)[:, None]).to(getattr(torch, dtype))
    qw = quantized(torch, readout, torch.randn(outputs, n, generator=gen, device="cuda"))
    qx = quantized(torch, readout, x)
    vx, vw = torch.empty(rows, n, device="cuda"), torch.empty(outputs, n, device="cuda")
    readout.mx_dequantize(*qx, vx)
    readout.mx_dequantize(*qw, vw)
    out = torch.full((rows, outputs), float("nan"), dtype=x.dtype, device="cuda")
    ws = torch.full((readout.mx_linear_workspace_bytes(rows, n),), 255, dtype=torch.uint8, device="cuda")
    readout.mx_linear(x, *qw, out, ws)
    vx, vw = vx.double(), vw.double()
    want = vx @ vw.t()
    bound = (n / 128 + 8) * U32 * (vx.abs() @ vw.abs().t()) + (U16 if dtype == "bfloat16" else U32) * want.abs() * 1.01
    assert float(((out.double() - want).abs() - bound).max()) <= 0
    again = torch.full_like(out, float("nan"))
    readout.mx_linear(x, *qw, again, ws)
    assert torch.equal(again, out)
