"""Builds the HIP libraries in-tree (hipcc, gfx950 only).  `python -m paper_2605_10905_amd.build`."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libattn_mi355x.so")
SOURCES = ["attn_api.hip", "attn_fwd_sp.hip", "attn_fwd_fp8.hip", "attn_bwd_bf16.hip", "gemm_api.hip", "gemm_bf16.hip", "gemm_wavek.hip"]
# what stands around attention in a layer (include/kv.h) is a library of its own: who only attends does not load it
LIB_KV = os.path.join(HERE, "libkv_mi355x.so")
SOURCES_KV = ["kv_api.hip", "rope.hip", "kv_decode.hip"]
CALL_KV = os.path.join(HERE, "_kv_call" + sysconfig.get_config_var("EXT_SUFFIX"))  # its Python side: host code, by the host compiler, for this Python
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# packed fp32 VALU forms are switched off on purpose (they have misbehaved on the test machines)
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument", "-Wno-inline-asm"]
# the one-wave-per-SIMD backward kernel keeps its score accumulators in ordinary registers, where the vector work reads them.
# (An internal switch of the compiler: known to the clang 22 of ROCm 7.2.0, with which all figures were taken.  A compiler that does not know
# it refuses the build; without it the kernels' register plan does not hold, and the listing has to be read anew for the wait states.)
# kv_decode.hip, one wave per SIMD too: its products in ordinary registers save 90 register moves a tile.  Calls without / with it, us: 1 x 500 keys
# 8.4 / 8.2, 24 ragged up to 1500, d = 64 21.6 / 21.0, 32 up to 9000, e4m3 67.7 / 66.3; groups of 64 queries, 64 x 4000 46.3 / 44.7, e4m3 35.3 / 31.6.
# Nothing there depends on it.
SOURCE_FLAGS = {"attn_bwd_bf16.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"], "kv_decode.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def _start(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    return cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(cmd, pr, verbose):
    out, _ = pr.communicate()
    out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
    if pr.returncode != 0:
        raise RuntimeError("the compiler failed:\n" + " ".join(cmd) + "\n" + out)
    if verbose and out.strip():
        print(out)


def _call_commands():
    """Compiling and linking the Python side of include/kv.h, or what is missing for it: the libraries are built without it."""
    try:
        import torch
    except ImportError:
        return None, "torch"
    where = os.path.dirname(torch.__file__)
    inc, python = os.path.join(where, "include"), sysconfig.get_path("include")
    if shutil.which("g++") is None:
        return None, "g++"
    for header in (os.path.join(python, "Python.h"), os.path.join(inc, "torch", "csrc", "autograd", "python_variable.h")):
        if not os.path.exists(header):
            return None, header
    obj = os.path.join(CSRC, "kv_call.o")
    compile_ = ["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DBUILT_FOR_TORCH="{torch.__version__}"', "-w",
                "-I", inc, "-I", os.path.join(inc, "torch", "csrc", "api", "include"), "-I", python, "-c", os.path.join(CSRC, "kv_call.cpp"), "-o", obj]
    link = ["g++", "-shared", obj, "-o", CALL_KV, f"-L{HERE}", "-lkv_mi355x", f"-L{os.path.join(where, 'lib')}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN"]
    return (compile_, link), ""


def build(verbose: bool = True, extra_flags=()) -> str:
    objs = {src: os.path.join(CSRC, src.replace(".hip", ".o")) for src in SOURCES + SOURCES_KV}
    procs = [_start([HIPCC, *FLAGS, *SOURCE_FLAGS.get(src, []), *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj], verbose) for src, obj in objs.items()]
    call, missing = _call_commands()
    host = _start(call[0], verbose) if call else None
    if os.path.exists(CALL_KV):
        os.remove(CALL_KV)  # (never beside a library of another build)
    for cmd, pr in procs:
        _finish(cmd, pr, verbose)
    for lib, sources in ((LIB, SOURCES), (LIB_KV, SOURCES_KV)):
        _finish(*_start([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *[objs[src] for src in sources], "-o", lib], verbose), verbose)
    if host is None:
        print(f"the Python side of include/kv.h is not built: {missing} is missing", file=sys.stderr)
        return LIB
    _finish(*host, verbose)
    _finish(*_start(call[1], verbose), verbose)
    return LIB


if __name__ == "__main__":
    build(extra_flags=sys.argv[1:])
