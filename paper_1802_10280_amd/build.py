"""Builds libescoin.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libescoin.so")

SOURCES = ["host.cpp", "plan.cpp", "pad_in.hip", "sconv_direct.hip", "sconv_tiled.hip", "mfma_plan.cpp", "sconv_mfma.hip", "pair_plan.cpp", "sconv_pair.hip", "sconv_first.hip",
           "linear_plan.cpp", "linear_few.hip", "linear_many.hip", "norm.hip"]

# Packed-FP32 VALU forms are switched off for every device translation unit.
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-x", "hip",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def _run(cmd: list[str], verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = ("is not a recognized feature for this target", "argument unused during compilation")
    err = "\n".join(l for l in res.stderr.splitlines() if not any(n in l for n in noise))
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err, file=sys.stderr)


def build(verbose: bool = False, extra: list[str] | None = None) -> str:
    """Compiles every source, a few side by side, and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp:
        objects = {s: os.path.join(tmp, s + ".o") for s in SOURCES}
        with ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            jobs = [pool.submit(_run, [hipcc, *flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC, *(extra or []), "-c", "-o", o,
                                       os.path.join(CSRC, s)], verbose) for s, o in objects.items()]
            for j in jobs:
                j.result()
        _run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB, *objects.values()], verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
