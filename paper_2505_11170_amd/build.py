"""Build ``libgws.so`` (HIP, gfx950 only) in-tree with hipcc.

    python -m paper_2505_11170_amd.build [--force]

hipcc cross-compiles without a GPU.  Floating-point contraction is off (the block
scale must be one defined sequence of fp32 operations) and packed-fp32 code
generation is disabled.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
SOURCES = ["gws_api.hip", "gws_sample.hip", "gws_linear.hip", "gws_gemm_stream.hip", "gws_gemm_stream_tn.hip", "gws_gemm128.hip", "gws_gemm256.hip", "gws_gemm256_tn.hip",
           "gws_gated_api.hip", "gws_gated.hip", "gws_gated256.hip", "gws_gated128.hip", "gws_gated_stream.hip", "gws_act8.hip",
           "gws_layer_api.hip", "gws_norm.hip", "gws_dense.hip", "gws_dense128.hip", "gws_dense256.hip", "gws_dense_stream.hip", "gws_adamw.hip"]
HEADERS = ["gws_device.h", "gws_launch.h", "gws_sample_tile.h", "gws_gemm256_core.h", "gws_gemm_stream_core.h", "gws_check.h", "gws_gated.h", "gws_gated_out.h",
           "gws_norm.h", "gws_dense.h", "gws_dense_out.h", "gws_adamw.h", "gws_gemm128_core.h", "gws_gemm_stream_kernel.h"]
OUT = os.path.join(_HERE, "libgws.so")

FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-mllvm", "-amdgpu-kernarg-preload-count=16",   # plain kernel arguments arrive in scalar registers
         "-Wall", "-Wno-unused-command-line-argument"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def stale() -> bool:
    if not os.path.exists(OUT):
        return True
    t = os.path.getmtime(OUT)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(_ROOT, "include", "gws.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return OUT
    bdir = os.path.join(_HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    inc = ["-I", os.path.join(_ROOT, "include"), "-I", CSRC]
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(bdir, src.replace(".hip", ".o"))
        cmd = [hipcc(), *FLAGS, *inc, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for cmd, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + out)
        if verbose and out.strip():
            print(out)
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", OUT, *objs]
    subprocess.run(cmd, check=True)
    return OUT


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose=True))
