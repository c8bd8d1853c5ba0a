"""Build the HIP library in-tree: paper_2404_04541_amd/libspgemm_gfx950.so."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(_HERE, "csrc", "spgemm_api.hip")
SRC_ATTENTION = os.path.join(_HERE, "csrc", "attention_api.hip")
LIB = os.path.join(_HERE, "libspgemm_gfx950.so")
LIB_CLOCKS = os.path.join(_HERE, "libspgemm_gfx950_clocks.so")   # the same sources with -DSPG_PHASE_CLOCKS (profiling only)

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-munsafe-fp-atomics",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def _hipcc(args: list, verbose: bool) -> None:
    cmd = ["hipcc", *FLAGS, *args]
    if verbose:
        print(" ".join(cmd))
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)


def build_library(verbose: bool = False, phase_clocks: bool = False) -> str:
    """Compile csrc/ for gfx950 with hipcc (cross-compiles without a GPU).  phase_clocks: the profiling
    variant whose dense kernels read the shader clock at phase boundaries (used by phase_profile.py only;
    the products alone)."""
    if phase_clocks:
        _hipcc(["-shared", "-DSPG_PHASE_CLOCKS=1", "-o", LIB_CLOCKS, SRC], verbose)
        return LIB_CLOCKS
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(2) as pool:
        sources = (SRC, SRC_ATTENTION)
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources]
        list(pool.map(lambda so: _hipcc(["-c", "-o", so[1], so[0]], verbose), zip(sources, objects)))
        _hipcc(["-shared", "-o", LIB, *objects], verbose)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_library(verbose=True, phase_clocks=True))
