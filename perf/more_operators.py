"""Performance cases of a gated hidden layer under the dense readout: a program that trains it on a sparse network's rows,
clips its gradients with the readout's, and answers with weights held as 4-bit whole numbers with a scale a group.

A case's fields:
  op       "gated":    h = act(x wg^T) * (x wu^T), T rows of D features to H hidden values: the layer as it answers
           "train":    the same with its gradients to x, wg and wu from the gradient of h
           "clip":     a list of tensors scaled so that their common norm is at most `most`; "count" of them, the largest of
                       `values` values
           "grouped":  T rows of D features times V x D weights held in 4 bits, a scale (and with `offsets` an
                       offset) for each `group` values of a row
  dtype    "f32" or "bf16"; "mixed" (clip): both
  act      "silu" or "gelu" (by the error function). A step at zero (relu) is left to tests: in fp32 a sum next to zero
           falls on either side of it with the order it is taken in.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LARGEST = 6.7e12  # operations of the largest listed case
MOST_VALUES = 1 << 30  # of the largest listed list of gradients


def listed():
    return [
        # one row through a small layer: latency
        dict(name="gated-m1-n1024-h4096-bf16", op="gated", T=1, D=1024, H=4096, dtype="bf16", act="silu"),
        # an evaluation batch through the layer of the 4096-neuron network
        dict(name="gated-m2000-n4096-h16384-bf16", op="gated", T=2000, D=4096, H=16384, dtype="bf16", act="silu"),
        # few rows, small layer: launches and the weights' traffic
        dict(name="train-m64-n1024-h4096-bf16", op="train", T=64, D=1024, H=4096, dtype="bf16", act="silu"),
        # odd sizes throughout, fp32
        dict(name="train-m1021-n1000-h2047-f32", op="train", T=1021, D=1000, H=2047, dtype="f32", act="gelu"),
        # the largest step
        dict(name="train-m8192-n4096-h16384-bf16", op="train", T=8192, D=4096, H=16384, dtype="bf16", act="silu"),
        # the gradients of one small layer and its readout: latency
        dict(name="clip-3-n524288-f32", op="clip", count=3, values=524288, dtype="f32", most=1.0),
        # many tensors of all sizes and both types
        dict(name="clip-240-n1000003-mixed", op="clip", count=240, values=1000003, dtype="mixed", most=1.0),
        # the gradients of wide layers: memory
        dict(name="clip-16-n134217728-bf16", op="clip", count=16, values=134217728, dtype="bf16", most=1.0),
        # one row over a small label set, fp32: latency
        dict(name="grouped-m1-n1000-c1000-g32-f32", op="grouped", T=1, D=1000, V=1000, group=32, offsets=True, dtype="f32"),
        # one row answered by a wide readout: the weights' bytes
        dict(name="grouped-m1-n4096-c65536-g128-bf16", op="grouped", T=1, D=4096, V=65536, group=128, offsets=False, dtype="bf16"),
        # a few rows together
        dict(name="grouped-m16-n16384-c16384-g64-bf16", op="grouped", T=16, D=16384, V=16384, group=64, offsets=True, dtype="bf16"),
        # a scoring batch
        dict(name="grouped-m2000-n4096-c16384-g128-bf16", op="grouped", T=2000, D=4096, V=16384, group=128, offsets=False, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over its logarithm: odd, even and round ones."""
    n = _log_int(rng, lo, hi)
    unit = rng.choice([1, 1, 40, 320])
    return n if n < 2 * unit else n // unit * unit


def draw(rng):
    op = rng.choice(["gated", "gated", "train", "train", "clip", "grouped", "grouped", "grouped"])
    while True:
        case = dict(op=op, dtype=rng.choice(["f32", "bf16"]))
        if op == "clip":
            case |= dict(count=_log_int(rng, 1, 300), values=_log_int(rng, 100, 1 << 27), dtype=rng.choice(["f32", "bf16", "mixed"]), most=rng.choice([1.0, 1.0, 1e6]))
            if sum(_clip_sizes(case)) <= MOST_VALUES // 2:
                return case
            continue
        case |= dict(T=_log_int(rng, 1, 8192), D=_size(rng, 64, 16384))
        if op == "grouped":
            case |= dict(V=_size(rng, 10, 65536), group=rng.choice([32, 64, 128]), offsets=rng.choice([False, True]))
            fits = case["D"] * case["V"] <= 1 << 28 and case["T"] * case["V"] <= 1 << 28
        else:
            case |= dict(H=_size(rng, 16, 32768), act=rng.choice(["silu", "gelu"]))
            fits = case["D"] * case["H"] <= 1 << 27 and case["T"] * case["H"] <= 1 << 27
        if fits and work(case)["flops"] <= LARGEST:
            return case


def _clip_sizes(case):
    """The tensors' sizes: the largest, the rest spread below it over their logarithm for many tensors, near it for few."""
    rng = random.Random(case["count"] * 1000003 + case["values"])
    low = 1 if case["count"] > 32 else max(1, case["values"] // 4)
    return [case["values"]] + [_log_int(rng, low, case["values"]) for _ in range(case["count"] - 1)]


def _flat(case, dtypes):
    """Room for the clipped tensors: one buffer a type, and each tensor's part of it, on a multiple of 64 values."""
    sizes, used, at = _clip_sizes(case), {}, []
    for n, dt in zip(sizes, dtypes):
        at.append(used.get(dt, 0))
        used[dt] = at[-1] + -(-n // 64) * 64
    flat = {dt: torch.zeros(n, dtype=dt, device="cuda") for dt, n in used.items()}
    return list(flat.values()), [flat[dt][k:k + n] for n, dt, k in zip(sizes, dtypes, at)]


def _clip_dtypes(case):
    return [DTYPES[("f32", "bf16")[i % 2] if case["dtype"] == "mixed" else case["dtype"]] for i in range(case["count"])]


def _code_rows(V, D):
    step = max(1, (1 << 26) // D)
    return [min(step, V - r) for r in range(0, V, step)]


def _encode(w, group, offsets, dt):
    """Rows of w in 4 bits: two codes to a byte, the even value low; a group's scale and offset, rounded to `dt` before the
    codes are taken with them. Rows are padded to whole groups."""
    n, d = w.shape
    groups = -(-d // group)
    s = torch.nn.functional.pad(w, (0, groups * group - d)).reshape(n, groups, group)
    if offsets:
        low = s.amin(2)
        scale, offset = ((s.amax(2) - low) / 15.0).to(dt), low.to(dt)
    else:
        scale = (s.abs().amax(2) / 7.0).to(dt)
        offset = -8.0 * scale.float()
    by = scale.float()
    q = torch.round((s - offset.float()[:, :, None]) / torch.where(by > 0, by, 1.0)[:, :, None]).clamp(0, 15).to(torch.uint8).reshape(n, -1)
    return (q[:, 0::2] | q[:, 1::2] << 4).contiguous(), scale, offset if offsets else None


def _inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    if case["op"] == "clip":
        # gradients: each tensor of its own size of values
        return {"tensors": [(rand(n) * 0.02 * (1 + i % 5)).to(dt) for i, (n, dt) in enumerate(zip(_clip_sizes(case), _clip_dtypes(case)))]}
    T, D, dt = case["T"], case["D"], DTYPES[case["dtype"]]
    # rows as the network leaves them: non-negative, many zeros, limited at 32
    s = {"x": (2.0 * rand(T, D) - 0.5).clamp(0.0, 32.0).to(dt)}
    if case["op"] == "grouped":
        parts = [_encode(rand(n, D) / math.sqrt(D), case["group"], case["offsets"], dt) for n in _code_rows(case["V"], D)]
        s["codes"], s["scales"] = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
        s["offsets"] = torch.cat([p[2] for p in parts]) if case["offsets"] else None
        return s
    H = case["H"]
    s["wg"], s["wu"] = ((rand(H, D) / math.sqrt(D)).to(dt) for _ in range(2))
    if case["op"] == "train":
        s["dh"] = (rand(T, H) / T).to(dt)  # of a mean over the rows
    return s


def prepare(case, seed):
    """The inputs, and the buffers for answers and scratch that a program keeps."""
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if case["op"] == "clip":
        s["flat"], s["out"] = _flat(case, _clip_dtypes(case))
        s["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
    elif case["op"] == "grouped":
        s["out"] = torch.empty(case["T"], case["V"], dtype=s["x"].dtype, device="cuda")
    else:
        s["h"] = torch.empty(case["T"], case["H"], dtype=s["x"].dtype, device="cuda")
        if case["op"] == "train":
            s["gate"], s["up"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])  # kept from the layer to its gradient
            s["dx"], s["dwg"], s["dwu"] = (torch.empty_like(s[k]) for k in ("x", "wg", "wu"))
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
    if c["op"] == "clip":
        ws = _workspace(s, readout.clip_workspace_bytes(c["count"]))
        readout.clip(s["tensors"], c["most"], s["norm"], ws, out=s["out"], stream=stream)
        return {"norm": s["norm"], "out": s["flat"]}
    x = s["x"]
    if c["op"] == "grouped":
        ws = _workspace(s, readout.grouped_linear_workspace_bytes(c["T"], c["V"], c["D"], x.dtype))
        readout.grouped_linear(x, s["codes"], s["scales"], s["out"], ws, group=c["group"], offsets=s["offsets"], stream=stream)
        return {"out": s["out"]}
    train = c["op"] == "train"
    ws = _workspace(s, readout.gated_workspace_bytes(c["T"], c["H"], c["D"], x.dtype, gradient=train))
    if not train:
        readout.gated(x, s["wg"], s["wu"], s["h"], ws, activation=c["act"], stream=stream)
        return {"h": s["h"]}
    kept = dict(gate=s["gate"], up=s["up"], activation=c["act"], stream=stream)
    readout.gated(x, s["wg"], s["wu"], s["h"], ws, **kept)
    readout.gated_gradient(x, s["wg"], s["wu"], s["dh"], s["dx"], s["dwg"], s["dwu"], ws, **kept)
    return {k: s[k] for k in ("h", "dx", "dwg", "dwu")}


def _plain(s):
    c = s["case"]
    if c["op"] == "clip":
        norm = torch.stack([t.double().square().sum() for t in s["tensors"]]).sum().sqrt()
        by = torch.clamp(c["most"] / norm, max=1.0).float()
        for t, o in zip(s["tensors"], s["out"]):
            o.copy_(t.float() * by)
        return {"norm": norm.float()[None], "out": s["flat"]}
    x = s["x"].float()
    if c["op"] == "grouped":
        codes, scales = s["codes"], s["scales"].float()
        q = torch.stack([codes & 15, codes >> 4], 2).reshape(c["V"], -1, c["group"]).float()
        w = q * scales[:, :, None] + s["offsets"].float()[:, :, None] if c["offsets"] else (q - 8.0) * scales[:, :, None]
        return {"out": (x @ w.reshape(c["V"], -1)[:, : c["D"]].t()).to(s["x"].dtype)}
    wg, wu, dt = s["wg"].float(), s["wu"].float(), s["x"].dtype
    g, u = x @ wg.t(), x @ wu.t()
    if c["act"] == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        act, slope = g * p, p * (1.0 + g * (1.0 - p))
    else:
        p = 0.5 * torch.special.erfc(g * -math.sqrt(0.5))
        act, slope = g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    h = (act * u).to(dt)
    if c["op"] == "gated":
        return {"h": h}
    dh = s["dh"].float()
    dg, du = dh * u * slope, dh * act
    return {"h": h, "dx": (dg @ wg + du @ wu).to(dt), "dwg": (dg.t() @ x).to(dt), "dwu": (du.t() @ x).to(dt)}


def work(case):
    if case["op"] == "clip":
        n = sum(k * t.itemsize for k, t in zip(_clip_sizes(case), _clip_dtypes(case)))
        return {"bytes": 2.0 * n + 4.0, "flops": 3.0 * sum(_clip_sizes(case))}
    size, T, D = DTYPES[case["dtype"]].itemsize, case["T"], case["D"]
    if case["op"] == "grouped":
        V, groups = case["V"], -(-D // case["group"])
        return {"bytes": size * T * (D + V) + 0.5 * V * D + size * V * groups * (2.0 if case["offsets"] else 1.0), "flops": 2.0 * T * V * D}
    H = case["H"]
    if case["op"] == "gated":
        return {"bytes": size * (T * (D + H) + 2.0 * H * D), "flops": 4.0 * T * H * D}
    return {"bytes": size * (2.0 * T * (D + H) + 4.0 * H * D), "flops": 12.0 * T * H * D}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "clip":
        total = 0.0
        for t in s["tensors"]:
            total += float(torch.linalg.vector_norm(t, dtype=torch.float64)) ** 2
        norm = math.sqrt(total)
        by = min(1.0, case["most"] / norm) if norm > 0 else 1.0
        norm64 = torch.tensor([norm], dtype=torch.float64, device="cuda")
        kinds = list(dict.fromkeys(_clip_dtypes(case)))
        if sum(_clip_sizes(case)) > 1 << 29:  # values of 8 bytes, all at once: the norm alone
            return {"norm": norm64, "out": [None for _ in kinds]}
        flat = []
        for kind in kinds:
            parts = [torch.nn.functional.pad(t.double() * by, (0, -t.numel() % 64)) for t in s["tensors"] if t.dtype == kind]
            flat.append(torch.cat(parts))
        return {"norm": norm64, "out": flat}
    x = s["x"].double()
    T, D = x.shape
    if case["op"] == "grouped":
        V, group, r = case["V"], case["group"], 0
        out = torch.empty(T, V, dtype=torch.float64, device="cuda")
        for n in _code_rows(V, D):
            at = slice(r, r + n)
            w = torch.empty(n, 2 * s["codes"].shape[1], dtype=torch.float64, device="cuda")
            w[:, 0::2] = s["codes"][at].double() % 16
            w[:, 1::2] = torch.floor(s["codes"][at].double() / 16)
            scale = s["scales"][at].double().repeat_interleave(group, 1)
            if case["offsets"]:
                w = w * scale + s["offsets"][at].double().repeat_interleave(group, 1)
            else:
                w = (w - 8) * scale
            out[:, at] = torch.mm(x, w[:, :D].t())
            r += n
        return {"out": out}
    wg, wu = s["wg"].double(), s["wu"].double()
    g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
    if case["act"] == "silu":
        p = torch.sigmoid(g)
        slope = p + g * p * torch.sigmoid(-g)
    else:
        p = torch.special.ndtr(g)
        slope = p + g * torch.exp(g.square() / -2) / math.sqrt(2 * math.pi)
    act = g * p
    if case["op"] == "gated":
        return {"h": act * u}
    dh = s["dh"].double()
    dg, du = dh * slope * u, dh * act
    return {"h": act * u, "dx": torch.mm(dg, wg) + torch.mm(du, wu), "dwg": torch.mm(dg.t(), x), "dwu": torch.mm(du.t(), x)}
