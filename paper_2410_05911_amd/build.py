"""Builds libaecct.so (host library + gfx950 kernels) in the package directory with hipcc.

Flags: -O3 for gfx950 only; -ffp-contract=off so that only the multiply-adds written as
fmaf are fused; packed fp32 instructions disabled; no fast-math (fp32 division and square
root stay correctly rounded, denormals are kept).
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libaecct.so")
SOURCES = ["host.cpp", "host_fused.cpp", "aap.cpp", "kernels_layered.hip", "kernel_fused.hip", "arith_check.hip", "spe.hip",
           "train.hip", "train_host.cpp", "norm.hip", "norm_host.cpp", "update.hip", "update_host.cpp",
           "linear.hip", "linear_f32.hip", "linear_bf16.hip", "linear_f16.hip", "linear_i8.hip", "linear_e4m3.hip", "linear_host.cpp",
           "dropout.hip", "dropout_host.cpp", "attention.hip", "attention_grad.hip",
           "attention_host.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

COMMON = ["-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Wall", "-Wno-unused-function",
          "-I", os.path.join(os.path.dirname(HERE), "include")]
DEVICE = ["-x", "hip", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def build(verbose: bool = False, jobs: int = 4) -> str:
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
        cmd = [HIPCC] + COMMON + DEVICE + ["-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        text = out.decode(errors="replace")
        text = "\n".join(ln for ln in text.splitlines() if "packed-fp32-ops" not in ln)
        if text.strip() and (verbose or p.returncode):
            print(text, file=sys.stderr)
        if p.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError(f"hipcc failed for {failed}")
    cmd = [HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB + ".tmp"] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
