"""Builds the HIP libraries in-tree (hipcc, gfx950 only).  `python -m paper_2605_10905_amd.build`."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libattn_mi355x.so")
SOURCES = ["attn_api.hip", "attn_fwd_sp.hip", "attn_fwd_fp8.hip", "attn_bwd_bf16.hip", "gemm_api.hip", "gemm_bf16.hip", "gemm_wavek.hip"]
# what stands around attention in a layer (include/kv.h) is a library of its own: who only attends does not load it
LIB_KV = os.path.join(HERE, "libkv_mi355x.so")
SOURCES_KV = ["kv_api.hip", "rope.hip", "kv_decode.hip"]
CALL_KV = os.path.join(HERE, "_kv_call.so")  # its Python side: host code, by the host compiler
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# packed fp32 VALU forms are switched off on purpose (they have misbehaved on the test machines)
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", "-Wno-inline-asm"]
# the one-wave-per-SIMD backward kernel keeps its score accumulators in ordinary registers, where the vector work reads them.
# (An internal switch of the compiler: known to the clang 22 of ROCm 7.2.0, with which all figures were taken.  A compiler that does not know
# it refuses the build; without it the kernels' register plan does not hold, and the listing has to be read anew for the wait states.)
# kv_decode.hip, one wave per SIMD too: its products in ordinary registers save 90 register moves a tile (16 x 2000 keys 25.7 -> 25.3 us,
# 1 x 500 4.8 -> 4.4); nothing there depends on it.
SOURCE_FLAGS = {"attn_bwd_bf16.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"], "kv_decode.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def build(verbose: bool = True, extra_flags=()) -> str:
    objs = {}
    procs = []
    for src in SOURCES + SOURCES_KV:
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        cmd = [HIPCC, *FLAGS, *SOURCE_FLAGS.get(src, []), *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs[src] = obj
    import sysconfig

    import torch

    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-w",
           "-I", inc, "-I", os.path.join(inc, "torch", "csrc", "api", "include"), "-I", sysconfig.get_path("include"),
           "-c", os.path.join(CSRC, "kv_call.cpp"), "-o", os.path.join(CSRC, "kv_call.o")]
    if verbose:
        print(" ".join(cmd), flush=True)
    procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, pr in procs:
        out, _ = pr.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if pr.returncode != 0:
            raise RuntimeError("the compiler failed:\n" + " ".join(cmd) + "\n" + out)
        if verbose and out.strip():
            print(out)
    for lib, sources in ((LIB, SOURCES), (LIB_KV, SOURCES_KV)):
        cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *[objs[src] for src in sources], "-o", lib]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
    tlib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-shared", os.path.join(CSRC, "kv_call.o"), "-o", CALL_KV, f"-L{HERE}", "-lkv_mi355x", f"-L{tlib}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    build(extra_flags=sys.argv[1:])
