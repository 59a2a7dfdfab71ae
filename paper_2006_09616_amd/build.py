"""Build step of the HIP library (hipcc, gfx950)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

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

FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
         # no packed FP32 instructions anywhere in the device code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # m0 on a clobber list is meant
         "-Wno-inline-asm",
         "-Rpass-analysis=kernel-resource-usage", "-fno-caret-diagnostics", "-I", os.path.join(ROOT, "include")]


def scratch_of(lines, source: str) -> list:
    """The kernels of a source that the compiler's remarks give scratch memory, with its bytes a lane."""
    name, found = "?", []
    for l in lines:
        if source not in l or ": remark: " not in l:
            continue
        text = l.split(": remark: ")[1].split(" [-R")[0].strip()
        if text.startswith("Function Name:"):
            name = text.split(":", 1)[1].strip()
        if text.startswith("ScratchSize") and text.split(":")[1].strip() != "0":
            found.append(f"{name}: {text}")
    return found


def build(verbose: bool = False, profile: bool = False) -> str:
    out = OUT_PROFILE if profile else OUT
    tmp = out + ".tmp"
    flags = [*FLAGS, *(["-DDTR_PROFILE"] if profile else [])]
    with tempfile.TemporaryDirectory() as where:
        objects = [os.path.join(where, os.path.basename(s) + ".o") for s in SOURCES]
        commands = [["hipcc", *flags, "-c", "-o", o, s] for o, s in zip(objects, SOURCES)]
        if verbose:
            print("\n".join(" ".join(c) for c in commands), flush=True)
        with ThreadPoolExecutor(len(commands)) as pool:
            results = list(pool.map(lambda c: subprocess.run(c, capture_output=True, text=True), commands))
        lines = [l for r in results for l in r.stderr.splitlines()]
        noise = [l for l in lines if l.strip() and "packed-fp32-ops" not in l and ": remark: " not in l]
        if any(r.returncode for r in results):
            raise RuntimeError("hipcc failed:\n" + "\n".join(noise))
        spilled = scratch_of(lines, "attention.hip")
        if spilled:
            # attention's loads into LDS are not the compiler's: a build that put
            # registers into scratch memory beside them has given wrong gradients
            raise RuntimeError("attention kernels use scratch memory:\n" + "\n".join(spilled))
        if verbose and noise:
            print("\n".join(noise), file=sys.stderr)
        link = ["hipcc", "-fPIC", "-shared", f"--offload-arch={ARCH}", "-o", tmp, *objects]
        if verbose:
            print(" ".join(link), flush=True)
        res = subprocess.run(link, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stderr)
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
