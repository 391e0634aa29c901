"""Weights of 4 bits on the GPU where a group's values or their differences reach the ends of fp32's range, or where its range is
far smaller than its values.

Bounds. A code is the nearest where its value is as near as any other's, but for the roundings of a difference and of a
quotient of at most 16 steps, 2^-24 of them each: 2^-19 steps either way, 2^-18 between two codes' distances."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_grouped import parts_of

pytestmark = pytest.mark.gpu
MOST = {"float32": (2.0 - 2.0 ** -23) * 2.0 ** 127, "bfloat16": (2.0 - 2.0 ** -7) * 2.0 ** 127}


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


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_ranges_far_smaller_than_their_values(group, dtype):
    """With offsets: the scale is (max - min) / 15, off by at most 2^-24 of it where the two are within a factor of two, their
    difference exact; else by the roundings of two quotients, together at most three times the difference's size, and of their
    difference: 4 * 2^-24. bf16 rounds once more, by 2^-8."""
    torch = torch_cuda()
    log(f"grouped narrow range {group} {dtype}")
    dt, gen = getattr(torch, dtype), torch.Generator("cuda").manual_seed(group)
    lows = [1.0, -1.0, 1000.0, -1000.0, 1e6, -1e6, 1e30, -1e30, 1e-30, -1e-30, 2.0 ** 127, -(2.0 ** 127)]
    widths = [2.0 ** -k for k in ((23, 22, 21, 20, 16, 10, 7, 5, 2, 1) if dtype == "float32" else (7, 6, 5, 4, 3, 2, 1))] + [0.0, 0.9]
    low = torch.tensor(lows, device="cuda").repeat_interleave(len(widths))[:, None]
    width = torch.tensor(widths, device="cuda").repeat(len(lows))[:, None]
    near = torch.rand(low.shape[0], 200, generator=gen, device="cuda")
    near[:, ::32] = 0.0
    near[:, 1::32] = 1.0
    w = (low + low * width * near).to(dt)
    (q, s, o), out, scales = quantised(w, group, True)
    wide = torch.nn.functional.pad(w.double(), (0, scales.shape[1] * group - 200), value=float("nan")).reshape(w.shape[0], -1, group)
    there = ~wide.isnan()
    top, bottom = torch.where(there, wide, -torch.inf).amax(2), torch.where(there, wide, torch.inf).amin(2)
    want = (top - bottom) / 15
    unit = 2.0 ** -22 + (2.0 ** -8 if dtype == "bfloat16" else 0.0)
    assert bool((want > 0).any()) and bool(((scales.double() - want).abs() <= unit * want).all())
    assert_nearest(torch, w, q, s, o)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offsets", [False, True])
def test_the_largest_numbers_are_read_back_finite(offsets, dtype):
    """Groups whose largest magnitudes are the largest numbers of the type and those below them: within half a step and the
    roundings of the scale (15 times 2^-8 of a step, twice where the next scale below is taken) and of the result."""
    torch = torch_cuda()
    log(f"grouped largest {offsets} {dtype}")
    dt, most = getattr(torch, dtype), MOST[dtype]
    last = 2.0 ** (127 - (7 if dtype == "bfloat16" else 23))  # the largest numbers' last place
    tops = torch.tensor([most - k * last for k in range(120)], dtype=torch.float64, device="cuda")
    w = torch.zeros(360, 64, dtype=torch.float64, device="cuda")
    w[:120, 0], w[120:240, 0], w[240:, 0] = tops, -tops, most
    w[:240:3, 1] = -w[:240:3, 0]
    w[240:, 1] = -most * (torch.arange(120, dtype=torch.float64, device="cuda") / 120)  # offsets far from the largest number
    w[:, 2] = w[:, 0] / 3
    w[:, 40] = w[:, 0] * 0.9
    w[1::2, 41] = -w[1::2, 40]
    w = w.to(dt)
    assert bool(w.isfinite().all()) and float(w.abs().max()) == most
    for group in (32, 64):
        (q, s, o), out, _ = quantised(w, group, offsets)
        assert bool(out.isfinite().all())
        unit = 2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -22
        assert bool(((out.double() - w.double()).abs() <= (0.5 + 30 * unit) * s + unit * w.double().abs()).all())
