"""Weights of 4 bits on the GPU where a group's values or their differences reach the ends of fp32's range.

Bounds. A code is the nearest where its value is as near as any other's, but for the roundings of a difference and of a
quotient of at most 16 steps, 2^-24 of them each: 2^-19 steps either way, 2^-18 between two codes' distances."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_grouped import parts_of

pytestmark = pytest.mark.gpu


def quantised(w, group, offsets):
    """Codes' numbers, scales and offsets of every weight in 64 bits, the values read back, and the scales."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    rows, n = w.shape
    groups = readout.grouped_groups(n, group)
    codes = torch.zeros(rows, groups * group // 2, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(rows, groups, dtype=w.dtype, device="cuda")
    low = torch.zeros_like(scales) if offsets else None
    out = torch.empty_like(w)
    readout.grouped_quantize(w, codes, scales, group=group, offsets=low)
    readout.grouped_dequantize(codes, scales, out, group=group, offsets=low)
    return parts_of(codes, scales, low, n, group), out, scales


def assert_nearest(torch, w, q, s, o):
    w = w.double()
    far = (q * s + o - w).abs()
    best = torch.stack([(c * s + o - w).abs() for c in range(16)]).amin(0)
    assert bool((far <= best + 2.0 ** -18 * s).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_ranges_past_the_largest_number(group, dtype):
    """With offsets: values on both sides whose difference to the smallest is no fp32 number."""
    torch = torch_cuda()
    log(f"grouped wide range {group} {dtype}")
    gen = torch.Generator("cuda").manual_seed(group)
    w = ((2 * torch.rand(50, 300, generator=gen, device="cuda") - 1) * 3.3e38).to(getattr(torch, dtype))
    w[0, :4] = torch.tensor([-3e38, 3e38, 1e38, 5e37])
    w[1] = w[1].clamp(min=-1e30)
    w[2, 5:] = 0.0
    (q, s, o), out, _ = quantised(w, group, True)
    assert bool(out.isfinite().all())
    assert_nearest(torch, w, q, s, o)
