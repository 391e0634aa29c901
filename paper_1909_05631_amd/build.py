"""Build libsdnn.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB_PATH = os.path.join(HERE, "libsdnn.so")
SOURCES = [os.path.join(HERE, "csrc", name)
           for name in ("library.hip", "readout.hip", "orthogonalize.hip", "mx.hip", "gated.hip", "clip.hip", "grouped.hip")]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # packed fp32 instructions are kept out of every kernel
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # fp32 semantics: no contraction beyond the explicit fmaf calls, IEEE denormals
    "-ffp-contract=off", "-fno-gpu-flush-denormals-to-zero",
    "-Wall", "-Wno-unused-result",
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    return os.path.join(rocm, "bin", "hipcc")


def _run(cmd: list[str]) -> str:
    res = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (res.stdout + res.stderr).splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{out}")
    return out


def build(verbose: bool = False) -> str:
    """Compile the sources side by side, link them, put the library in place."""
    with tempfile.TemporaryDirectory() as objects:
        def compile_one(source: str) -> tuple[str, str]:
            obj = os.path.join(objects, os.path.basename(source) + ".o")
            return obj, _run([hipcc(), *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-c", source, "-o", obj])

        with concurrent.futures.ThreadPoolExecutor(len(SOURCES)) as pool:
            made = list(pool.map(compile_one, SOURCES))
        tmp = LIB_PATH + ".tmp"
        out = [o for _, o in made]
        out.append(_run([hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *[obj for obj, _ in made]]))
    if verbose and "".join(out).strip():
        print("\n".join(o for o in out if o.strip()))
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
