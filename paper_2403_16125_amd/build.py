"""Build the HIP library libarena.so in-tree for gfx950 (hipcc)."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "_build", "libarena.so")
SOURCES = [os.path.join(CSRC, "arena_host.cpp"), os.path.join(CSRC, "arena_kernels.hip"),
           os.path.join(CSRC, "arena_sched.hip"), os.path.join(CSRC, "arena_proxy.hip"),
           # layer operators (include/arena_layer.h)
           os.path.join(CSRC, "arena_layer_host.cpp"), os.path.join(CSRC, "arena_gemm_bf16.hip"),
           os.path.join(CSRC, "arena_gemm_f16.hip"), os.path.join(CSRC, "arena_norm.hip"),
           os.path.join(CSRC, "arena_update.hip"),
           # layers of experts and the vocabulary's loss (include/arena_experts.h, include/arena_loss.h)
           os.path.join(CSRC, "arena_experts_host.cpp"), os.path.join(CSRC, "arena_groups_bf16.hip"),
           os.path.join(CSRC, "arena_groups_f16.hip"), os.path.join(CSRC, "arena_route.hip"),
           os.path.join(CSRC, "arena_loss_host.cpp"), os.path.join(CSRC, "arena_loss_bf16.hip"),
           os.path.join(CSRC, "arena_loss_f16.hip"), os.path.join(CSRC, "arena_loss.hip")]

VALU_RATE_SRC = os.path.join(CSRC, "valu_rate.hip")
VALU_RATE_OUT = os.path.join(PKG, "_build", "libvalu_rate.so")   # fp64-vs-fp32 issue-rate microbenchmark

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                      # keep the operation order of the formulas
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def build(verbose: bool = False) -> str:
    """Compiles every source anew (side by side) and links the library."""
    out = os.path.dirname(OUT)
    os.makedirs(out, exist_ok=True)
    objects = [os.path.join(out, os.path.basename(src) + ".o") for src in SOURCES]
    compile_flags = [f for f in FLAGS if f != "-shared"]
    with concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        jobs = [pool.submit(_run, [HIPCC] + compile_flags + ["-c", "-o", obj, src], verbose)
                for src, obj in zip(SOURCES, objects)]
        for job in jobs:
            job.result()
    tmp = OUT + ".tmp"
    _run([HIPCC] + FLAGS + ["-o", tmp] + objects, verbose)
    os.replace(tmp, OUT)
    for obj in objects:
        os.remove(obj)
    tmp = VALU_RATE_OUT + ".tmp"
    _run([HIPCC] + FLAGS + ["-o", tmp, VALU_RATE_SRC], verbose)
    os.replace(tmp, VALU_RATE_OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)
