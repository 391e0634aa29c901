"""The orthogonalisation of matrices that one workgroup's LDS does not hold: the form of several launches, with A's k whole and
in parts, wide and tall, alone and in batches, against 64 bits."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import MUON, U16, newton_schulz, orth_bound, sum_bound

pytestmark = pytest.mark.gpu

# wide, tall; A in parts of a long side; blocks of every size; batches
SHAPES = [(3, 200, 330), (3, 330, 200), (1, 150, 6000), (1, 6000, 150), (2, 140, 900), (2, 900, 140), (2, 257, 255), (4, 161, 128), (5, 128, 161), (40, 200, 200), (8, 700, 900), (8, 900, 700),
          (1, 1300, 1300)]


def is_large(rows, cols):
    """The documented limit of the one-launch form: both factors in 4 bytes a value, sides padded to 32, in 152 KB."""
    m, n = (-(-v // 32) * 32 for v in sorted((rows, cols)))
    return m > 128 or (m * n + m * m) * 4 > 152 * 1024


def space(readout, torch, *shape):
    return torch.full((readout.orthogonalize_workspace_bytes(*shape),), 255, dtype=torch.uint8, device="cuda")


def inputs(torch, shape, seed, dtype="float32"):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_large(shape, dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize large {shape} {dtype}")
    assert is_large(*shape[1:])
    g = inputs(torch, shape, shape[1], dtype)
    out = torch.full_like(g, float("nan"))
    ws = space(readout, torch, *shape)
    for steps, coef in ((5, MUON), (0, MUON), (1, MUON), (2, MUON), (8, (1.875, -1.25, 0.375))):
        readout.orthogonalize(g, out, ws, steps=steps, coefficients=coef)
        want = newton_schulz(torch, g, steps, coef, 1e-7, torch.float64)
        plain = newton_schulz(torch, g, steps, coef, 1e-7, torch.float32)
        for b in range(shape[0]):  # each matrix by itself
            bound = orth_bound(g[b], plain[b], want[b]) + (U16 * float(want[b].norm()) if dtype == "bfloat16" else 0)
            assert float((out[b].double() - want[b]).norm()) <= bound, (steps, coef, b)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(3, 200, 330), (3, 330, 200), (2, 150, 1501), (2, 1501, 150), (2, 301, 301)])
def test_strides_and_in_place(shape, dtype):
    """Views into NaN, apart and unaligned, give the contiguous form's bits and touch nothing around; so does each alone."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize large strides {shape} {dtype}")
    batch, rows, cols = shape
    assert is_large(rows, cols)
    for before, after in ((2, 1), (1, 2), (8, 8)):
        flat = torch.full((batch, rows + 2, before + cols + after), float("nan"), device="cuda").to(getattr(torch, dtype))
        g = flat[:, 1:rows + 1, before:before + cols]
        g.copy_(inputs(torch, shape, 8))
        nans = int(flat.isnan().sum())
        dense = g.contiguous()
        want = torch.empty_like(dense)
        ws = space(readout, torch, *shape)
        readout.orthogonalize(dense, want, ws)
        for steps in (0, 5):
            other = torch.full_like(flat, float("nan"))
            readout.orthogonalize(g, other[:, 1:rows + 1, before:before + cols], ws, steps=steps)
            assert int(other.isnan().sum()) == nans
            if steps:
                assert torch.equal(other[:, 1:rows + 1, before:before + cols], want)
        readout.orthogonalize(g, g, ws)
        assert torch.equal(g, want) and int(flat.isnan().sum()) == nans


@pytest.mark.parametrize("shape", [(2, 200, 330), (2, 330, 200), (1, 150, 6000)])
@pytest.mark.parametrize("scale", [1e-30, 1e-9, 1e-4, 1e6, 1e25])
def test_scales(scale, shape):
    """Any size of update: the norm neither overflows nor vanishes; one far below eps only grows by a, step by step. The
    matrices of a batch have sizes of their own."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize large scale {scale} {shape}")
    assert is_large(*shape[1:])
    g = scale * inputs(torch, shape, 2)
    if shape[0] > 1:
        g[1] *= 1e-8
    out = torch.empty_like(g)
    readout.orthogonalize(g, out, space(readout, torch, *shape), eps=1e-7)
    want = newton_schulz(torch, g, 5, MUON, 1e-7, torch.float64)
    for b in range(shape[0]):
        # from 2^-20 a product and its sums' roundings, at most fourfold a step; below the normal numbers, their quantum
        bound = 4 * (2.0 ** -20 + sum_bound(max(shape[1:]))) * float(want[b].norm()) + 2.0 ** -149 * want[b].numel() ** 0.5
        assert float((out[b].double() - want[b]).norm()) <= bound


@pytest.mark.parametrize("shape", [(4, 200, 330), (4, 330, 200), (4, 150, 1500)])
def test_zeros_and_not_finite(shape):
    """A matrix of zeros gives zeros, one with a NaN NaN, and neither touches the others of the batch."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize large zeros, NaN {shape}")
    assert is_large(*shape[1:])
    g = inputs(torch, shape, 2)
    ws = space(readout, torch, *shape)
    good, out = torch.empty_like(g), torch.empty_like(g)
    readout.orthogonalize(g, good, ws)
    g[0] = 0
    g[2, 3, 4] = float("nan")
    readout.orthogonalize(g, out, ws)
    assert not out[0].any() and bool(out[2].isnan().all()) and torch.equal(out[1], good[1]) and torch.equal(out[3], good[3])


@pytest.mark.parametrize("shape", [(2, 200, 330), (1, 150, 6000), (2, 330, 200)])
def test_streams_and_graph(shape):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"orthogonalize large graph {shape}")
    assert is_large(*shape[1:])
    g = inputs(torch, shape, 3)
    out, want = torch.empty_like(g), torch.empty_like(g)
    ws = space(readout, torch, *shape)
    readout.orthogonalize(g, want, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    readout.orthogonalize(g, out, ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
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
