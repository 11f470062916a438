"""Builds the HIP library ``libgd.so`` for gfx950 next to this file.

Every source is compiled by ``hipcc`` with IEEE-exact float settings: no
fast-math, no contraction into fused multiply-adds, denormals kept, and the
packed-fp32 instructions switched off.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libgd.so")
SOURCES = ["gd_select.hip", "gd_sampled.hip", "gd_dense.hip", "gd_layout.hip", "gd_cand.hip", "gd_direct.hip", "gd_quant.hip", "gd_apply.hip", "gd_api.hip", "gd_static.hip",
           "gd_norm.hip", "gd_adamw.hip", "gd_linear.hip", "gd_gemm_bf16.hip", "gd_gemm_f16.hip", "gd_gemm_f32.hip"]
HEADERS = ["gd_device.hpp", "gd_kernels.h", "gd_internal.h", "gd_host.hpp", "gd_ops.hpp", "gd_gemm.hpp",
           "gd_gemm_launch.hpp"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-ffp-contract=off",
    "-fno-fast-math",
    "-fno-gpu-rdc",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
    "-Wno-unused-result",
]


def build(verbose: bool = False, out: str = LIB, extra_flags=(), objdir: str = "") -> str:
    """Compile every source and link ``out`` (default ``libgd.so`` here); returns its path.

    ``extra_flags`` go on every compile and the link line (a test build with
    host-only sanitizers uses it); such a build belongs in its own ``objdir``.
    """
    objdir = objdir or os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(src: str) -> str:
        obj = os.path.join(objdir, src + ".o")
        cmd = [HIPCC, *FLAGS, *extra_flags, "-I", INCLUDE, "-I", CSRC, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and r.stderr.strip():
            print(r.stderr, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = out + f".tmp{os.getpid()}"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *extra_flags, *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build(verbose=True))
