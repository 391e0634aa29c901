"""What the binding of the dense readout's operators takes and refuses, beyond the C ABI's own checks."""
import pytest

from tests.gpu_util import log, torch_cuda

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(0, 4, 5), (0, 300, 200)])
def test_no_matrices_are_no_error(shape):
    """As the C ABI has it: a batch of none is nothing to do."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"no matrices {shape}")
    g = torch.empty(*shape, device="cuda")
    ws = torch.empty(max(1, readout.orthogonalize_workspace_bytes(*shape)), dtype=torch.uint8, device="cuda")
    readout.orthogonalize(g, torch.empty_like(g), ws)
    with pytest.raises(ValueError):
        readout.orthogonalize(g[:, :0], g[:, :0], ws)  # matrices without rows


def test_orthogonalize_refuses_what_is_no_tensor():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("no tensor")
    g = torch.zeros(2, 4, 5, device="cuda")
    ws = torch.empty(readout.orthogonalize_workspace_bytes(2, 4, 5), dtype=torch.uint8, device="cuda")
    for out in (None, 3, g.tolist(), g.cpu(), g[0]):
        with pytest.raises(ValueError):
            readout.orthogonalize(g, out, ws)


@pytest.mark.parametrize("rows,outputs", [(0, 5), (5, 0)])
def test_no_rows_or_outputs_of_4_bits(rows, outputs):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"mx {rows} x {outputs}")
    x = torch.randn(rows, 40, device="cuda")
    nb = readout.mx_blocks(40)
    codes, scales = torch.zeros(outputs, 16 * nb, dtype=torch.uint8, device="cuda"), torch.zeros(outputs, nb, dtype=torch.uint8, device="cuda")
    xc, xs = torch.zeros(rows, 16 * nb, dtype=torch.uint8, device="cuda"), torch.zeros(rows, nb, dtype=torch.uint8, device="cuda")
    out = torch.empty(rows, outputs, device="cuda")
    ws = torch.empty(max(1, readout.mx_linear_workspace_bytes(rows, 40)), dtype=torch.uint8, device="cuda")
    readout.mx_quantize(x, xc, xs)
    readout.mx_dequantize(xc, xs, torch.empty_like(x))
    readout.mx_product(xc, xs, codes, scales, 40, out)
    readout.mx_linear(x, codes, scales, out, ws)
