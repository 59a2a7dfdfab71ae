"""Build step of the HIP library (hipcc, gfx950)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
SOURCES = [os.path.join(CSRC, f) for f in ("dtr_sim.cpp", "dtr_log.cpp", "replay.hip", "replay_log.hip",
                                            "dtr_ops.cpp", "attention.hip", "rows.hip")]
OUT = os.path.join(HERE, "libdtrsim.so")
# the same sources with the in-kernel cycle timers (profile.py); never the product
OUT_PROFILE = os.path.join(HERE, "libdtrsim_prof.so")
# the operators on torch tensors (C++ over the library's C ABI)
OPS_SOURCE = os.path.join(CSRC, "ops_torch.cpp")
OPS_OUT = os.path.join(HERE, "_ops.so")
ARCH = "gfx950"

FLAGS = ["-O3", "-std=c++17", "-fPIC", "-shared", f"--offload-arch={ARCH}",
         # no packed FP32 instructions anywhere in the device code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include")]


def build(verbose: bool = False, profile: bool = False) -> str:
    out = OUT_PROFILE if profile else OUT
    tmp = out + ".tmp"
    cmd = ["hipcc", *FLAGS, *(["-DDTR_PROFILE"] if profile else []), "-o", tmp, *SOURCES]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = [l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l and l.strip()]
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(noise))
    if verbose and noise:
        print("\n".join(noise), file=sys.stderr)
    os.replace(tmp, out)
    return out


def build_ops(verbose: bool = False) -> str:
    """The torch binding of the operators; links against libdtrsim.so beside it."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension as ext
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    libs = ext.library_paths()
    tmp = OPS_OUT + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[f for p in [*ext.include_paths(), os.path.join(rocm, "include"), sysconfig.get_paths()["include"]]
             for f in ("-isystem", p)],
           "-o", tmp, OPS_SOURCE, *["-L" + p for p in [*libs, HERE]], "-l:libdtrsim.so", "-lc10", "-lc10_hip", "-ltorch_cpu",
           "-ltorch_hip", "-ltorch", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stderr)
    os.replace(tmp, OPS_OUT)
    return OPS_OUT


if __name__ == "__main__":
    print(build(verbose=True))
    print(build_ops(verbose=True))
