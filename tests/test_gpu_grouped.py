"""Weights of 4 bits with group scales on the GPU: quantisation against its definition, products against 64 bits.

Bounds. u16 = 2^-8 and u32 = 2^-24 are the unit roundoffs of bf16 and fp32. A product is a sum over groups of
s sum x q + o sum x, o = -8 s without offsets: exact products (of fp32 x in three parts too), in a chain of at most k / 16 sums
of 32 products, one for each group, and a few where waves meet; off by at most (k / 16 + 60) u32 times sum |x| (|s| q + |o|)
with q at most 15. Where the weights are written as values of x's type first, each is off by u |w| and the two roundings of
its product and sum in fp32, products of fp32 values in two parts by 4 * 2^-22 and 2^-38 of the largest magnitudes, and
their sum by (k / 4 + 40) u32. The result is rounded once."""
import math

import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_readout import assert_within, matrix

pytestmark = pytest.mark.gpu
U16, U32 = 2.0 ** -8, 2.0 ** -24


def parts_of(codes, scales, offsets, n, group):
    """q, scale and offset of every weight, in 64 bits."""
    import torch
    q = torch.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1)[:, :n].double()
    s = scales.double().repeat_interleave(group, 1)[:, :n]
    o = -8 * s if offsets is None else offsets.double().repeat_interleave(group, 1)[:, :n]
    return q, s, o


def few(rows, outputs, n, fp32):
    """Rows whose groups' sums are scaled, by the header's rule."""
    return rows <= 64 or (outputs >= 4096 and outputs * n >= 1 << 24 and rows <= (256 if fp32 else 128))


def reference(x, codes, scales, offsets, group):
    n, fp32 = x.shape[1], x.element_size() == 4
    unit = U32 if fp32 else U16
    q, s, o = parts_of(codes, scales, offsets, n, group)
    x = x.double()
    w = q * s + o
    value = x @ w.t()
    size = x.abs() @ (15 * s.abs() + o.abs()).t()
    e = (n / 16 + 60) * U32 * size
    if not few(*x.shape[:1], codes.shape[0], n, fp32):
        m = x.abs() @ w.abs().t()
        e = 2 * U32 * size + unit * m + (n / 4 + 40) * U32 * m
        if fp32:
            e += 4 * 2.0 ** -22 * m + 2.0 ** -38 * n * x.abs().max() * w.abs().max()
    return value, e + unit * (value.abs() + e)


class Weights:
    def __init__(self, rows, n, group, offsets, dtype, seed=0):
        from paper_1909_05631_amd import readout
        torch = torch_cuda()
        gen = torch.Generator("cuda").manual_seed(seed)
        dt, groups = getattr(torch, dtype), readout.grouped_groups(n, group)
        self.codes = torch.randint(0, 256, (rows, groups * group // 2), generator=gen, device="cuda", dtype=torch.uint8)
        self.scales = (0.1 + torch.rand(rows, groups, generator=gen, device="cuda")).div(4 * math.sqrt(n)).to(dt)
        self.offsets = (torch.rand(rows, groups, generator=gen, device="cuda") - 1.0).div(math.sqrt(n)).to(dt) if offsets else None
        self.n, self.group = n, group


SHAPES = [(1, 1, 1), (1, 10, 31), (2, 17, 33), (3, 300, 1000), (4, 16, 128), (5, 33, 129), (15, 1000, 65), (16, 129, 4096), (17, 40, 300), (31, 9000, 70), (48, 100, 1024), (64, 257, 520),
          (65, 40, 64), (100, 300, 1000), (193, 193, 97), (300, 1000, 250), (1000, 70, 513), (1, 20000, 200), (1, 40, 20001), (16, 30, 16384), (7, 50, 40000), (300, 250, 4000), (65, 4100, 4100),
          (128, 4096, 4096), (129, 4097, 4099), (256, 4096, 4096), (257, 4100, 4100), (100, 4095, 4200)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,outputs,n", SHAPES)
def test_linear(rows, outputs, n, dtype):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    for group in readout.GROUPS:
        for offsets in (False, True):
            log(f"grouped {rows} x {n} to {outputs} in {group} {offsets} {dtype}")
            w = Weights(outputs, n, group, offsets, dtype, seed=rows)
            dt = getattr(torch, dtype)
            x = matrix(torch, torch.Generator("cuda").manual_seed(n), rows, n, dt)
            out = torch.full((rows, outputs), 7.0, dtype=dt, device="cuda")
            ws = torch.full((readout.grouped_linear_workspace_bytes(rows, outputs, n, dt),), 255, dtype=torch.uint8, device="cuda")
            readout.grouped_linear(x, w.codes, w.scales, out, ws, group=group, offsets=w.offsets)
            assert_within("out", out, reference(x, w.codes, w.scales, w.offsets, group))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (8, 0), (3, 5), (24, 8)])
def test_strides_and_alignment(pad, offset, dtype):
    """Rows apart from each other, bases on any value, NaN all around."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"grouped strides {pad} {offset} {dtype}")
    dt = getattr(torch, dtype)
    gen = torch.Generator("cuda").manual_seed(5)
    for rows, outputs, n in ((3, 70, 96), (9, 45, 131), (70, 141, 97), (250, 210, 98)):
        w = Weights(outputs, n, 32, True, dtype)
        x, out = matrix(torch, gen, rows, n, dt, 1.0, pad, offset), matrix(torch, gen, rows, outputs, dt, 1.0, pad, offset)
        around = out.as_strided((out.untyped_storage().nbytes() // out.element_size(),), (1,), 0)
        before = around.isnan().sum()
        ws = torch.empty(max(1, readout.grouped_linear_workspace_bytes(rows, outputs, n, dt)), dtype=torch.uint8, device="cuda")
        readout.grouped_linear(x, w.codes, w.scales, out, ws, group=32, offsets=w.offsets)
        assert_within("out", out, reference(x, w.codes, w.scales, w.offsets, 32))
        assert around.isnan().sum() == before


@pytest.mark.parametrize("rows", [1, 16, 33, 100])
def test_rows_do_not_meet(rows):
    """A row of x that is not finite, or a group that stands for NaN, reaches its own row or output alone; the codes behind
    the last value reach nothing."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"grouped not finite {rows}")
    for dtype in ("float32", "bfloat16"):
        dt, n, outputs = getattr(torch, dtype), 140, 50
        w = Weights(outputs, n, 32, False, dtype)
        x = torch.randn(rows, n, device="cuda").to(dt)
        ws = torch.empty(max(1, readout.grouped_linear_workspace_bytes(rows, outputs, n, dt)), dtype=torch.uint8, device="cuda")

        def run():
            out = torch.empty(rows, outputs, dtype=dt, device="cuda")
            readout.grouped_linear(x, w.codes, w.scales, out, ws, group=32)
            return out

        want = run()
        w.codes[:, n // 2:] ^= 0xFF
        assert torch.equal(run(), want)
        w.scales[7, 4] = float("nan")
        got = run()
        keep = [i for i in range(outputs) if i != 7]
        assert bool(got[:, 7].isnan().all()) and torch.equal(got[:, keep], want[:, keep])
        for bad in (float("nan"), float("inf")):
            x[rows // 2, 99] = bad
            got = run()
            rest = [i for i in range(rows) if i != rows // 2]
            assert not bool(got[rows // 2].isfinite().any())
            assert torch.equal(got[rest][:, keep], want[rest][:, keep])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n,pad,offset", [(1, 1, 0, 0), (2, 31, 0, 0), (3, 33, 2, 1), (4, 128, 0, 0), (5, 129, 8, 8), (64, 1000, 0, 0), (7, 4096, 0, 3), (1000, 65, 0, 0)])
def test_quantize(rows, n, pad, offset, group, dtype):
    """Scales and offsets to the bit, codes the nearest: by the definition in fp32, whose divisions are rounded correctly on
    both sides. The values that they stand for are one fp32 product and sum, rounded."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"grouped quantise {rows} x {n} in {group} {dtype}")
    dt, gen = getattr(torch, dtype), torch.Generator("cuda").manual_seed(rows)
    w = matrix(torch, gen, rows, n, dt, 1.0, pad, offset)
    w[0, 0] = 0.0
    if rows > 4:
        w[1], w[2], w[3] = 0.0, w[2].abs(), -w[3].abs()
        w[4] = 1.5
    groups = readout.grouped_groups(n, group)
    for offsets in (False, True):
        codes = torch.full((rows, groups * group // 2), 255, dtype=torch.uint8, device="cuda")
        scales = torch.full((rows, groups), 7.0, dtype=dt, device="cuda")
        low = torch.full_like(scales, 7.0) if offsets else None
        readout.grouped_quantize(w, codes, scales, group=group, offsets=low)
        wide = torch.nn.functional.pad(w.float().cpu(), (0, groups * group - n), value=float("nan")).reshape(rows, groups, group)
        there = ~wide.isnan()
        top, bottom = torch.where(there, wide, -math.inf).amax(2), torch.where(there, wide, math.inf).amin(2)
        s = (top / 15 - bottom / 15 if offsets else torch.maximum(top, -bottom) / 7).to(dt)
        assert torch.equal(scales.cpu(), s)
        o = bottom.to(dt) if offsets else torch.zeros_like(s)
        if offsets:
            assert torch.equal(low.cpu(), o)
        by = torch.where(s > 0, s, 1.0).float()[:, :, None]
        q = torch.round((wide - o.float()[:, :, None]) / by)
        q = q.clamp(0, 15) if offsets else q.clamp(-8, 7) + 8
        q = torch.where(s.float()[:, :, None] > 0, q, 0.0 if offsets else 8.0)
        got = torch.stack([codes & 15, codes >> 4], 2).reshape(rows, -1)[:, :n].cpu()
        want = torch.where(there, q, 0.0).reshape(rows, -1)[:, :n].to(torch.uint8)
        assert torch.equal(got, want)
        out = matrix(torch, gen, rows, n, dt, 1.0, pad, offset)
        around = out.as_strided((out.untyped_storage().nbytes() // out.element_size(),), (1,), 0)
        before = around.isnan().sum()
        readout.grouped_dequantize(codes, scales, out, group=group, offsets=low)
        qd, sd, od = parts_of(codes, scales, low, n, group)
        value = qd * sd + od
        assert_within("out", out, (value, 2 * U32 * (qd * sd.abs() + od.abs()) + (U32 if dtype == "float32" else U16) * value.abs()))
        assert around.isnan().sum() == before
        # half a step (of 15 to the group's range), and the rounding of the scale and offset
        far = (out.double() - w.double()).abs()
        unit = U32 if dtype == "float32" else U16
        assert bool((far <= 0.5 * sd + 16 * unit * (15 * sd + od.abs() + w.double().abs())).all())


def test_quantize_special_values():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("grouped special values")
    for dtype in (torch.float32, torch.bfloat16):
        w = torch.zeros(6, 64, dtype=dtype, device="cuda")
        w[1, 3], w[2, 40], w[3, 5] = float("nan"), float("inf"), -float("inf")
        w[4, :2] = torch.tensor([3e38, -3e38])
        w[5, :2] = torch.tensor([1e-45, -1e-45])
        for offsets in (False, True):
            codes = torch.zeros(6, 32, dtype=torch.uint8, device="cuda")
            scales = torch.zeros(6, 2, dtype=dtype, device="cuda")
            low = torch.zeros_like(scales) if offsets else None
            out = torch.empty_like(w)
            readout.grouped_quantize(w, codes, scales, group=32, offsets=low)
            readout.grouped_dequantize(codes, scales, out, group=32, offsets=low)
            bad = out.isnan()
            assert bool(bad[1, :32].all()) and bool(bad[2, 32:].all()) and bool(bad[3, :32].all()) and int(bad.sum()) == 96
            assert not out[0].any() and bool(out[4].isfinite().all())
            assert float((out[4].double() - w[4].double()).abs().max()) <= 0.6 * float(scales[4, 0])
            assert float(out[5].double().abs().max()) <= 2e-45


@pytest.mark.parametrize("rows", [1, 40, 200])
def test_stream_and_graph(rows):
    """The same bits on another stream and in a graph that is replayed on changing rows."""
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"grouped graph {rows}")
    for dtype in ("float32", "bfloat16"):
        dt = getattr(torch, dtype)
        w = Weights(700, 1000, 64, True, dtype)
        x = torch.randn(rows, 1000, device="cuda").to(dt)
        out, got = (torch.zeros(rows, 700, dtype=dt, device="cuda") for _ in range(2))
        ws = torch.empty(max(1, readout.grouped_linear_workspace_bytes(rows, 700, 1000, dt)), dtype=torch.uint8, device="cuda")
        run = lambda to, stream=None: readout.grouped_linear(x, w.codes, w.scales, to, ws, group=64, offsets=w.offsets, stream=stream)  # noqa: E731
        run(out)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        run(got, side)
        side.synchronize()
        assert torch.equal(out, got)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(out, torch.cuda.current_stream())
        for k in range(4):
            x.mul_(0.5 + 0.25 * k)
            graph.replay()
            torch.cuda.synchronize()
            run(got, torch.cuda.current_stream())
            torch.cuda.synchronize()
            assert torch.equal(out, got), f"replay {k}"


@pytest.mark.parametrize("rows,outputs", [(0, 5), (5, 0)])
def test_no_rows_or_outputs(rows, outputs):
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log(f"grouped {rows} x {outputs}")
    x = torch.randn(rows, 40, device="cuda")
    codes, scales = torch.zeros(outputs, 32, dtype=torch.uint8, device="cuda"), torch.zeros(outputs, 2, device="cuda")
    ws = torch.empty(1, dtype=torch.uint8, device="cuda")
    readout.grouped_linear(x, codes, scales, torch.empty(rows, outputs, device="cuda"), ws, group=32)
    w = torch.empty(outputs, 40, device="cuda")
    readout.grouped_quantize(w, codes, scales, group=32)
    readout.grouped_dequantize(codes, scales, w, group=32)


def test_binding_refuses():
    from paper_1909_05631_amd import readout
    torch = torch_cuda()
    log("grouped refusals")
    x, c, s = torch.zeros(4, 100, device="cuda"), torch.zeros(7, 64, dtype=torch.uint8, device="cuda"), torch.zeros(7, 1, device="cuda")
    out, ws = torch.zeros(4, 7, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    good = dict(x=x, codes=c, scales=s, out=out, workspace=ws)
    readout.grouped_linear(**good)
    for bad in (dict(group=16), dict(group=32), dict(group="128"), dict(codes=c[:, :32]), dict(codes=c.int()), dict(codes=c[:6]), dict(codes=c[0]), dict(scales=s.bfloat16()), dict(scales=s[:, 0]),
                dict(offsets=s[:5]), dict(offsets=s.double()), dict(x=x.half()), dict(x=x[:, :30].t()), dict(out=out[:, :5]), dict(out=out.bfloat16()), dict(x=x.cpu()), dict(codes=c.cpu()),
                dict(workspace=ws.cpu()), dict(codes=c.t().contiguous().t()), dict(codes=None), dict(scales=None)):
        with pytest.raises(ValueError):
            readout.grouped_linear(**{**good, **bad})
    with pytest.raises(ValueError):
        readout.grouped_quantize(x, c, s)
    with pytest.raises(ValueError):
        readout.grouped_dequantize(c, s, x)
    many = torch.zeros(70, 100, device="cuda")
    with pytest.raises(readout.SdnnError) as e:
        readout.grouped_linear(many, c, s, torch.zeros(70, 7, device="cuda"), ws[:256])
    assert e.value.name == "SDNN_ERANGE"
