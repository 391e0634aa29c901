"""The dense readout's operators at the ends of their sizes: rows of 2^20 values, one row or column, many matrices."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import Case, MUON, U16, U32, newton_schulz, orth_bound, sum_bound

pytestmark = pytest.mark.gpu
LONG = 1 << 20


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,classes,features,pad", [(3, 5, LONG, 0), (200, 250, LONG, 0), (200, 150, LONG, 0), (200, 201, LONG - 1, 2), (70, 9, LONG, 500000)])
def test_long_rows(rows, classes, features, pad, dtype):
    log(f"readout long rows {rows} x {classes} x {features} + {pad} {dtype}")
    c = Case(rows, classes, features, dtype, seed=1, pad=pad)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(1, 1, LONG), (1, LONG, 1), (1, 3, LONG), (1, LONG, 3), (1, 130, LONG // 8), (1, LONG // 8, 130), (65535, 3, 5), (3000, 140, 130)])
def test_long_and_many_matrices(shape, dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize ends {shape} {dtype}")
    g = torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(getattr(torch, dtype))
    out = torch.full_like(g, float("nan"))
    ws = torch.full((readout.orthogonalize_workspace_bytes(*shape),), 255, dtype=torch.uint8, device="cuda")
    readout.orthogonalize(g, out, ws)
    some = [0, shape[0] // 2, shape[0] - 1]
    want = newton_schulz(torch, g[some], 5, MUON, 1e-7, torch.float64)
    plain = newton_schulz(torch, g[some], 5, MUON, 1e-7, torch.float32)
    for i, b in enumerate(some):
        bound = max(orth_bound(g[b], plain[i], want[i]), 4 * sum_bound(max(shape[1:])) * float(want[i].norm())) + (U16 * float(want[i].norm()) if dtype == "bfloat16" else 0)
        assert float((out[b].double() - want[i]).norm()) <= bound
    assert bool(out.isfinite().all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,outputs", [(1, 70), (1, 5000), (40, 300), (300, 1)])
def test_long_rows_of_4_bits(rows, outputs, dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"mx long rows {rows} x {outputs} {dtype}")
    gen = torch.Generator("cuda").manual_seed(3)
    for n in (LONG, LONG - 77):
        x = torch.randn(rows, n, generator=gen, device="cuda").to(getattr(torch, dtype))
        nb = readout.mx_blocks(n)
        codes, scales = (torch.randint(0, hi, (outputs, wide), dtype=torch.uint8, generator=gen, device="cuda") for hi, wide in ((256, 16 * nb), (254, nb)))
        scales.clamp_(120, 134)
        codes.view(outputs, -1)[:, (n + 1) // 2:] = 0
        if n % 2:
            codes[:, n // 2] &= 15
        out = torch.full((rows, outputs), float("nan"), dtype=x.dtype, device="cuda")
        ws = torch.full((readout.mx_linear_workspace_bytes(rows, n),), 255, dtype=torch.uint8, device="cuda")
        readout.mx_linear(x, codes, scales, out, ws)
        xc, xs = torch.empty(rows, 16 * nb, dtype=torch.uint8, device="cuda"), torch.empty(rows, nb, dtype=torch.uint8, device="cuda")
        readout.mx_quantize(x, xc, xs)
        vx, vw = torch.empty(rows, n, device="cuda"), torch.empty(min(outputs, 70), n, device="cuda")
        readout.mx_dequantize(xc, xs, vx)
        readout.mx_dequantize(codes[:70], scales[:70], vw)
        vx, vw = vx.double(), vw.double()
        want = vx @ vw.t()
        bound = (n / 128 + 8) * U32 * (vx.abs() @ vw.abs().t()) + (U16 if dtype == "bfloat16" else U32) * want.abs() * 1.01
        assert float(((out[:, :70].double() - want).abs() - bound).max()) <= 0 and bool(out.isfinite().all())
