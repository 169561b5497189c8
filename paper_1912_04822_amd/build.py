"""Compile the HIP library in-tree for gfx950 (``python -m paper_1912_04822_amd.build``)."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmolgrid_hip.so")
# the C++ side of the Python binding (host code only)
BINDING_SOURCE = os.path.join(CSRC, "mg_binding.cpp")
BINDING = os.path.join(HERE, "_binding.so")
# measurement build: the same sources with -DMG_TIMING_AIDS (kernel phases can be switched off
# to time the rest; such runs write wrong grids, so the release library has none of it)
LIB_TIMING = os.path.join(HERE, "libmolgrid_hip_timing.so")

# -ffp-contract=off: nothing is fused behind the code's back (the binary-mode
# predicate and the double-precision transform are specified operation by
# operation); fused multiply-adds are written as fmaf where wanted.
# packed FP32 instructions are switched off for the device code.
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off", "-fno-fast-math",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument", "-Wno-unknown-attributes",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def build_binding(verbose: bool = False) -> str:
    """Compile the C++ side of the Python binding against the installed torch."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    includes = cpp_extension.include_paths() + [sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI)]
    for path in includes:
        cmd += ["-isystem", path]
    cmd += [BINDING_SOURCE, "-o", BINDING, "-L" + os.path.join(os.path.dirname(torch.__file__), "lib"),
            "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("the binding does not compile:\n" + res.stdout + res.stderr)
    return BINDING


def build_library(verbose: bool = False, timing_aids: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    out = LIB_TIMING if timing_aids else LIB
    cmd = [hipcc] + HIPCC_FLAGS + (["-DMG_TIMING_AIDS"] if timing_aids else []) + ["-o", out] + sources()
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    msgs = "\n".join(l for l in (res.stdout + res.stderr).splitlines()
                     if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + msgs)
    if verbose and msgs.strip():
        print(msgs)
    if not timing_aids:
        build_binding(verbose)
    return out


if __name__ == "__main__":
    print(build_library(verbose=True, timing_aids="--timing-aids" in sys.argv[1:]))
    sys.exit(0)
