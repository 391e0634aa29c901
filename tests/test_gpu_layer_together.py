"""A step of training and an answer with all of the readout's operators in a row, as a program makes them: the gated layer,
the readout's loss and gradient, the layer's gradient, the common norm and the clipped gradients, an orthogonalised update;
then the trained weights in 4 bits, layer and readout. Each operator is checked against 64 bits on what the one before it
left, with its own bounds; the whole step is captured into a graph and replayed."""
import pytest

from tests.gpu_util import log, torch_cuda
from tests.test_gpu_clip import check as check_clip
from tests.test_gpu_gated import reference as layer_reference
from tests.test_gpu_grouped import reference as grouped_reference
from tests.test_gpu_readout import assert_within
from tests.test_gpu_readout import reference as loss_reference

pytestmark = pytest.mark.gpu


class Step:
    def __init__(self, rows, features, hidden, classes, dtype):
        from paper_1909_05631_amd import readout
        self.torch = torch = torch_cuda()
        self.r, dt = readout, getattr(torch, dtype)
        gen = torch.Generator("cuda").manual_seed(rows)
        rand = lambda *s, scale=1.0: (torch.randn(*s, generator=gen, device="cuda") * scale).to(dt)  # noqa: E731
        self.x = rand(rows, features).clamp(min=0)
        self.wg, self.wu, self.w = rand(hidden, features, scale=features ** -0.5), rand(hidden, features, scale=features ** -0.5), rand(classes, hidden, scale=hidden ** -0.5)
        self.y = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
        self.y[::9] = -1
        self.h, self.gate, self.up, self.dh = (torch.empty(rows, hidden, dtype=dt, device="cuda") for _ in range(4))
        self.loss, self.lse = (torch.empty(rows, device="cuda") for _ in range(2))
        self.grads = [torch.empty_like(t) for t in (self.wg, self.wu, self.w)]
        self.clipped = [torch.empty_like(t) for t in self.grads]
        self.update, self.norm = torch.empty_like(self.w), torch.empty(1, device="cuda")
        need = max(readout.gated_workspace_bytes(rows, hidden, features, dt), readout.workspace_bytes(rows, classes, hidden, dt), readout.clip_workspace_bytes(3),
                   readout.orthogonalize_workspace_bytes(1, classes, hidden))
        self.ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        self.most = 0.01

    def run(self, stream=None):
        r = self.r
        kept = dict(activation="silu", gate=self.gate, up=self.up, stream=stream)
        r.gated(self.x, self.wg, self.wu, self.h, self.ws, **kept)
        r.loss(self.h, self.w, self.y, self.loss, self.lse, self.ws, stream=stream)
        r.gradient(self.h, self.w, self.y, self.lse, self.dh, self.grads[2], self.ws, stream=stream)
        r.gated_gradient(self.x, self.wg, self.wu, self.dh, None, self.grads[0], self.grads[1], self.ws, **kept)
        r.clip(self.grads, self.most, self.norm, self.ws, out=self.clipped, stream=stream)
        r.orthogonalize(self.clipped[2], self.update, self.ws, stream=stream)

    def outputs(self):
        return [self.h, self.loss, self.lse, self.dh, *self.grads, self.norm, *self.clipped, self.update]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("sizes", [(5, 64, 48, 10), (90, 130, 100, 33), (300, 200, 260, 1000)])
def test_training_step(sizes, dtype):
    log(f"together {sizes} {dtype}")
    s = Step(*sizes, dtype)
    t = s.torch
    s.run()
    layer = layer_reference(t, "silu", s.x, s.wg, s.wu, s.dh)
    assert_within("h", s.h, layer[2])
    loss = loss_reference(t, s.h, s.w, s.y, None)
    live = s.y >= 0
    assert_within("loss", s.loss, loss[0])
    assert_within("lse", s.lse[live], tuple(v[live] for v in loss[1]))
    assert_within("dh", s.dh, loss[2])
    assert not s.dh[~live].any()
    for name, got, want in (("dwg", s.grads[0], layer[4]), ("dwu", s.grads[1], layer[5]), ("dw", s.grads[2], loss[3])):
        assert_within(name, got, want)
    check_clip(t, s.grads, s.clipped, s.norm, s.most)
    # rows without a label add nothing to any weight's gradient
    grads = [g.clone() for g in s.grads]
    s.x[~live] *= 3
    s.run()
    assert all(t.equal(a, b) for a, b in zip(s.grads, grads))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_step_in_a_graph(dtype):
    log(f"together graph {dtype}")
    s = Step(200, 130, 100, 300, dtype)
    t = s.torch
    s.run()
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        s.run(stream=t.cuda.current_stream())
    for k in range(4):
        s.x.mul_(0.5 + 0.25 * k)
        s.wg.add_(0.01)
        graph.replay()
        t.cuda.synchronize()
        got = [v.clone() for v in s.outputs()]
        for v in s.outputs():
            v.fill_(3)
        s.run(stream=t.cuda.current_stream())
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip(got, s.outputs())), f"replay {k}"


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [1, 40, 100])
def test_answer(rows, dtype):
    """The layer in x's type, the readout's weights in 4 bits."""
    log(f"together answer {rows} {dtype}")
    s = Step(rows, 130, 100, 300, dtype)
    t, r = s.torch, s.r
    groups = r.grouped_groups(100, 32)
    codes, scales = t.empty(300, groups * 16, dtype=t.uint8, device="cuda"), t.empty(300, groups, dtype=s.w.dtype, device="cuda")
    offsets, out = t.empty_like(scales), t.empty(rows, 300, dtype=s.w.dtype, device="cuda")
    ws = t.empty(max(1, r.grouped_linear_workspace_bytes(rows, 300, 100, s.w.dtype)), dtype=t.uint8, device="cuda")
    r.grouped_quantize(s.w, codes, scales, group=32, offsets=offsets)
    r.gated(s.x, s.wg, s.wu, s.h, s.ws)
    r.grouped_linear(s.h, codes, scales, out, ws, group=32, offsets=offsets)
    assert_within("out", out, grouped_reference(s.h, codes, scales, offsets, 32))
    # a weight is off by half a step at most, and by what its scale's and offset's rounding moves it
    unit = t.finfo(s.w.dtype).eps / 2
    step = scales.double().repeat_interleave(32, 1)[:, :100]
    far = s.h.double().abs() @ (step * (0.5 + 32 * unit) + 16 * unit * s.w.double().abs()).t()
    value, bound = grouped_reference(s.h, codes, scales, offsets, 32)
    assert bool(((value - s.h.double() @ s.w.double().t()).abs() <= far + bound).all())


def test_gate_or_up_alone_is_kept():
    log("together one kept")
    for rows in (3, 40, 300):
        s = Step(rows, 130, 100, 30, "float32")
        s.r.gated(s.x, s.wg, s.wu, s.h, s.ws, gate=s.gate, up=s.up)
        want = s.h.clone(), s.gate.clone(), s.up.clone()
        for name, i in (("gate", 1), ("up", 2)):
            getattr(s, name).fill_(5)
            s.h.fill_(5)
            s.r.gated(s.x, s.wg, s.wu, s.h, s.ws, **{name: getattr(s, name)})
            assert s.torch.equal(s.h, want[0]) and s.torch.equal(getattr(s, name), want[i])
