"""Performance cases of the dense readout's operators: a program that trains a readout on a sparse
network's rows, updates it and answers with it in 4 bits, as it calls the library.

A case's fields:
  op       "score":    the softmax cross entropy of T rows of D features over V classes, no gradient
           "train":    the loss and the gradients of its mean over the counted rows, to the rows and the weights
           "orth":     B matrices of R x C orthogonalised by Newton-Schulz products (a momentum, five steps)
           "linear":   T rows of D features times V x D weights held as microscaled 4-bit floats
           "quantize": T rows of D values to microscaled 4-bit floats and back
  dtype    "f32" (what the network writes) or "bf16" (a readout trained in 16 bits)
"""
from __future__ import annotations

import math

import torch

own = False

STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # the magnitudes of a 4-bit float with 2 exponent bits
LARGEST = 6.7e12  # operations of the largest listed case


def listed():
    return [
        # one row scored against a small label set: latency
        dict(name="score-m1-n1024-c1000-f32", op="score", T=1, D=1024, V=1000, dtype="f32"),
        # an evaluation batch over many classes, 16-bit
        dict(name="score-m2000-n4096-c16384-bf16", op="score", T=2000, D=4096, V=16384, dtype="bf16"),
        # ten digits read out of the 1024-neuron network's rows
        dict(name="train-m2000-n1024-c10-f32", op="train", T=2000, D=1024, V=10, dtype="f32"),
        # odd sizes throughout, fp32
        dict(name="train-m1021-n1000-c10007-f32", op="train", T=1021, D=1000, V=10007, dtype="f32"),
        # few rows, many classes: the weights' traffic counts
        dict(name="train-m64-n1024-c65536-bf16", op="train", T=64, D=1024, V=65536, dtype="bf16"),
        # the largest step
        dict(name="train-m8192-n4096-c32768-bf16", op="train", T=8192, D=4096, V=32768, dtype="bf16"),
        # small updates of several layers at once: latency
        dict(name="orth-b4-128x256-f32", op="orth", B=4, R=128, C=256, dtype="f32"),
        # an odd, tall update in 16 bits
        dict(name="orth-2000x1021-bf16", op="orth", B=1, R=2000, C=1021, dtype="bf16"),
        # a square update of the 4096-neuron width
        dict(name="orth-4096x4096-f32", op="orth", B=1, R=4096, C=4096, dtype="f32"),
        # one row answered by a wide readout: the weights' bytes
        dict(name="linear-m1-n4096-c65536-bf16", op="linear", T=1, D=4096, V=65536, dtype="bf16"),
        # a large scoring batch
        dict(name="linear-m4096-n16384-c16384-bf16", op="linear", T=4096, D=16384, V=16384, dtype="bf16"),
        # the rows of the 16384-neuron network compressed for keeping
        dict(name="quantize-m8192-n16384-f32", op="quantize", T=8192, D=16384, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over its logarithm: odd, even and round ones."""
    n = _log_int(rng, lo, hi)
    unit = rng.choice([1, 1, 40, 320])
    return n if n < 2 * unit else n // unit * unit


def draw(rng):
    op = rng.choice(["score", "train", "train", "orth", "orth", "linear", "linear", "quantize"])
    case = dict(op=op, dtype=rng.choice(["f32", "bf16"]))
    while True:
        if op == "orth":
            case |= dict(B=rng.choice([1, 1, 2, 5]), R=_size(rng, 16, 8192), C=_size(rng, 16, 8192))
        else:
            case |= dict(T=_log_int(rng, 1, 8192), D=_size(rng, 64, 16384))
            if op != "quantize":
                case["V"] = _size(rng, 10, 65536)
        # no dearer than the largest listed case, nor larger than it in memory
        if work(case)["flops"] <= LARGEST and case.get("T", 1) * case.get("V", 1) <= 1 << 28 and case.get("D", 1) * case.get("V", 1) <= 1 << 28:
            return case


def _encode(x, n):
    """Blocks of 32 along the rows (n values, padded to 128) as 4-bit codes and the scales' exponents."""
    pad = -(-n // 128) * 128
    s = torch.nn.functional.pad(x.float(), (0, pad - n)).reshape(x.shape[0], -1, 32)
    top = s.abs().amax(2, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(-127, 127)
    s = torch.ldexp(s, -e)
    a = s.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)
    return torch.copysign(q, s), e


def _pack(q, e):
    """Codes two to a byte, the even one low, and a byte a scale: exponent + 127."""
    a = q.abs()
    code = torch.zeros(a.shape, dtype=torch.uint8, device=a.device)
    for v in GRID[1:]:
        code += a >= v
    code += 8 * torch.signbit(q).to(torch.uint8)
    code = code.reshape(q.shape[0], -1)
    return (code[:, 0::2] | code[:, 1::2] << 4).contiguous(), (e.reshape(q.shape[0], -1) + 127).to(torch.uint8)


def _unpack(codes, scales):
    lut = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    q = lut[torch.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1).long()]
    return torch.ldexp(q.reshape(codes.shape[0], -1, 32), scales[:, :, None].int() - 127).reshape(codes.shape[0], -1)


def _inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    if case["op"] == "orth":
        B, R, C = case["B"], case["R"], case["C"]
        # a momentum: a few strong directions over noise
        return {"g": (0.02 * rand(B, R, C) + rand(B, R, 4) @ rand(B, 4, C) / math.sqrt(R)).to(dt)}
    T, D = case["T"], case["D"]
    # rows as the network leaves them: non-negative, many zeros, limited at 32
    s = {"x": (2.0 * rand(T, D) - 0.5).clamp(0.0, 32.0).to(dt)}
    if case["op"] in ("score", "train"):
        V = case["V"]
        s["w"] = (rand(V, D) / math.sqrt(D)).to(dt)
        y = torch.randint(0, V, (T,), generator=gen, device="cuda")
        if T > 1:  # rows without a label
            y = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.05, -1, y)
        s["y"] = y
    elif case["op"] == "linear":
        V = case["V"]
        s["codes"], s["scales"] = zip(*[_pack(*_encode(rand(n, D) / math.sqrt(D), D)) for n in _rows(V, D)])
        s["codes"], s["scales"] = torch.cat(s["codes"]), torch.cat(s["scales"])
    return s


def _rows(V, D):
    step = max(1, (1 << 26) // D)
    return [min(step, V - r) for r in range(0, V, step)]


def prepare(case, seed):
    """The inputs, and the buffers for answers and scratch that a program keeps."""
    s = _inputs(case, seed)
    s["case"] = dict(case)
    x = s["x"] if "x" in s else s["g"]
    if case["op"] in ("score", "train"):
        T = case["T"]
        s["loss"], s["lse"] = (torch.empty(T, dtype=torch.float32, device="cuda") for _ in range(2))
        if case["op"] == "train":
            s["dx"], s["dw"] = torch.empty_like(x), torch.empty_like(s["w"])
    elif case["op"] == "linear":
        s["out"] = torch.empty(case["T"], case["V"], dtype=x.dtype, device="cuda")
    else:
        s["out"] = torch.empty_like(x)
    if case["op"] == "quantize":
        nb = -(-case["D"] // 128) * 4
        s["codes"] = torch.empty(case["T"], 16 * nb, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(case["T"], nb, dtype=torch.uint8, device="cuda")
    s["workspace"] = torch.empty(0, dtype=torch.uint8, device="cuda")
    return s


def _workspace(s, need):
    """The program's scratch, made in its first pass."""
    if s["workspace"].numel() < need:
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s["workspace"]


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_1909_05631_amd import readout

    c, stream = s["case"], torch.cuda.current_stream()
    if c["op"] == "orth":
        g = s["g"]
        ws = _workspace(s, readout.orthogonalize_workspace_bytes(*g.shape))
        readout.orthogonalize(g, s["out"], ws, steps=STEPS, coefficients=COEF, eps=EPS, stream=stream)
        return {"out": s["out"]}
    x = s["x"]
    if c["op"] == "quantize":
        readout.mx_quantize(x, s["codes"], s["scales"], stream=stream)
        readout.mx_dequantize(s["codes"], s["scales"], s["out"], stream=stream)
        return {"out": s["out"]}
    if c["op"] == "linear":
        ws = _workspace(s, readout.mx_linear_workspace_bytes(c["T"], c["D"]))
        readout.mx_linear(x, s["codes"], s["scales"], s["out"], ws, stream=stream)
        return {"out": s["out"]}
    w, y = s["w"], s["y"]
    train = c["op"] == "train"
    ws = _workspace(s, readout.workspace_bytes(c["T"], c["V"], c["D"], x.dtype, gradient=train))
    readout.loss(x, w, y, s["loss"], s["lse"], ws, stream=stream)
    if not train:
        return {"loss": s["loss"], "lse": s["lse"]}
    readout.gradient(x, w, y, s["lse"], s["dx"], s["dw"], ws, stream=stream)
    return {"loss": s["loss"], "dx": s["dx"], "dw": s["dw"]}


def _plain(s):
    c = s["case"]
    if c["op"] == "orth":
        a, b, k = COEF
        x = s["g"].float()
        if c["R"] > c["C"]:
            x = x.mT.contiguous()
        x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
        for _ in range(STEPS):
            m = x @ x.mT.contiguous()
            x = a * x + (b * m + k * (m @ m)) @ x
        return {"out": (x.mT if c["R"] > c["C"] else x).to(s["g"].dtype)}
    x = s["x"]
    if c["op"] == "quantize":
        q, e = _encode(x, c["D"])
        return {"out": torch.ldexp(q, e).reshape(c["T"], -1)[:, : c["D"]].to(x.dtype)}
    if c["op"] == "linear":
        q, e = _encode(x, c["D"])
        return {"out": (torch.ldexp(q, e).reshape(c["T"], -1) @ _unpack(s["codes"], s["scales"]).t()).to(x.dtype)}
    x, w, y = s["x"].float(), s["w"].float(), s["y"]
    logit = x @ w.t()
    top = logit.amax(1, keepdim=True)
    p = torch.exp(logit - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    counted = y >= 0
    at = y.clamp(min=0)[:, None]
    loss = torch.where(counted, lse - logit.gather(1, at)[:, 0], 0.0)
    if c["op"] == "score":
        return {"loss": loss, "lse": lse}
    up = torch.where(counted, 1.0 / counted.sum().clamp(min=1).float(), 0.0)[:, None]
    p = p * (up / total)
    p.scatter_add_(1, at, -up)
    return {"loss": loss, "dx": (p @ w).to(s["x"].dtype), "dw": (p.t() @ x).to(s["w"].dtype)}


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "orth":
        m, n = sorted((case["R"], case["C"]))
        # two of the three products of a step are symmetric
        return {"bytes": 2.0 * size * case["B"] * m * n, "flops": float(STEPS) * case["B"] * (3.0 * m * m * n + 1.0 * m * m * m)}
    T, D = case["T"], case["D"]
    if case["op"] == "quantize":
        return {"bytes": 2.0 * size * T * D, "flops": 0.0}
    V = case["V"]
    if case["op"] == "linear":
        return {"bytes": size * T * (D + V) + V * D * 17.0 / 32.0, "flops": 2.0 * T * V * D}
    if case["op"] == "score":
        return {"bytes": size * (T + V) * D + 16.0 * T, "flops": 2.0 * T * V * D}
    return {"bytes": 2.0 * size * (T + V) * D + 12.0 * T, "flops": 6.0 * T * V * D}


def _exact_mx(x, n):
    """The values that rows of x stand for after quantisation, in 64 bits: each compared with the middles
    between neighbours of the grid (a tie goes to the neighbour of even code)."""
    x = torch.nn.functional.pad(x.double(), (0, -n % 32)).reshape(x.shape[0], -1, 32)
    top = x.abs().amax(2, keepdim=True)
    scale = torch.exp2(torch.where(top > 0, torch.floor(torch.log2(top)), -200.0).sub(2.0).clamp(-127.0, 127.0))
    a, q = x.abs() / scale, torch.zeros_like(x)
    for i in range(7):
        mid, gap = (GRID[i] + GRID[i + 1]) / 2, GRID[i + 1] - GRID[i]
        q += gap * ((a >= mid) if i % 2 else (a > mid))
    return (q * scale * torch.sign(x)).reshape(x.shape[0], -1)[:, :n]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "orth":
        a, b, c = COEF
        x = s["g"].double()
        x /= torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + EPS
        tall = case["R"] > case["C"]
        for _ in range(STEPS):  # p(X X^T) X = X p(X^T X): the smaller of the two products
            xt = x.transpose(1, 2).contiguous()
            m = torch.bmm(xt, x) if tall else torch.bmm(x, xt)
            k = c * torch.bmm(m, m)
            k.add_(m, alpha=b).diagonal(dim1=1, dim2=2).add_(a)
            x = torch.bmm(x, k) if tall else torch.bmm(k, x)
        return {"out": x}
    T, D = case["T"], case["D"]
    if case["op"] == "quantize":
        return {"out": _exact_mx(s["x"], D)}
    if case["op"] == "linear":
        V = case["V"]
        lut = torch.tensor(GRID, dtype=torch.float64, device="cuda")
        x = torch.nn.functional.pad(_exact_mx(s["x"], D), (0, -D % 128))
        out = torch.empty(T, V, dtype=torch.float64, device="cuda")
        r = 0
        for n in _rows(V, D):
            b = s["codes"][r:r + n].int()
            w = torch.empty(n, 2 * b.shape[1], dtype=torch.float64, device="cuda")
            for half in (0, 1):
                code = b >> 4 * half & 15
                w[:, half::2] = lut[code & 7] * (1 - 2 * (code >> 3))
            w *= torch.exp2(s["scales"][r:r + n].double() - 127).repeat_interleave(32, 1)
            out[:, r:r + n] = x @ w.t()
            r += n
        return {"out": out}
    x, w, y = s["x"].double(), s["w"].double(), s["y"]
    logit = x @ w.t()
    lse = torch.logsumexp(logit, 1)
    keep = torch.nonzero(y >= 0).flatten()
    loss = torch.zeros(T, dtype=torch.float64, device="cuda")
    loss[keep] = lse[keep] - logit[keep, y[keep]]
    if case["op"] == "score":
        return {"loss": loss, "lse": lse}
    g = torch.zeros_like(logit)
    g[keep] = torch.exp(logit[keep] - lse[keep, None])
    g[keep, y[keep]] -= 1.0
    g /= max(1, keep.numel())
    return {"loss": loss, "dx": g @ w, "dw": g.t() @ x}
