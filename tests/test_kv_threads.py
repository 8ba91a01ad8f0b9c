"""While a call of include/kv.h is inside the library, other Python threads run: a launch can wait for the device, and what it waits for
can need the interpreter.  Behind a runtime whose launch waits, for five seconds at most, until another thread has said something."""
import json
import os
import subprocess
import sys

import pytest

from tests.test_kv_abi import P, ROOT, ROPE

_RUNTIME = """
#define hipLaunchKernel recorded_launch
#include "launch_recorder.cpp"
#undef hipLaunchKernel
#include <atomic>
#include <chrono>
#include <thread>
static std::atomic<int> inside{0}, heard{0};
extern "C" {
int is_inside() { return inside; }
void say() { heard = 1; }
int hipLaunchKernel(const void* stub, Dim3 grid, Dim3 block, void** args, size_t shared, void* stream) {
  inside = 1;
  for (int i = 0; i < 5000 && !heard; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
  if (!heard) return error = 1;
  return recorded_launch(stub, grid, block, args, shared, stream);
}
}
"""

_MAIN = """
import ctypes, importlib, json, sys, threading, time
import torch
rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
kv = importlib.import_module("paper_2605_10905_amd.kv")
name, kw = json.load(sys.stdin)
over = threading.Event()

def other():
    while not rec.is_inside() and not over.is_set():
        time.sleep(0.001)
    rec.say()

t = threading.Thread(target=other)
t.start()
status = getattr(kv, name)(**kw, stream=0, check=False)
over.set()
t.join()
print(status)
"""

_BWD = dict(ROPE, dq=P, dk=P, dv=P, dqkv=P, dld=256, dq_weight=P, dk_weight=P, workspace=P, B=1, Hq=2, Hkv=1, N=8, d=64)
_PAGED = dict(k_cache=P, v_cache=P, pages=P, d=64, W=2, page_size=16, num_pages=9, dtype=0, Hkv=1, Hq=2)
CALLS = [("rope_qkv", dict(ROPE, q=P, k=P, v=P, B=1, Hq=2, Hkv=1, N=8, d=64)), ("rope_qkv_bwd", _BWD), ("kv_append", dict(ROPE, **_PAGED, seq=P, q=P, T=4, S=4)),
         ("kv_decode", dict(_PAGED, q=P, lens=P, o=P, lse=P, workspace=P, B=2, scale=0.1))]


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    at = tmp_path_factory.mktemp("runtime")
    (at / "waiting.cpp").write_text(_RUNTIME)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-pthread", "-I", os.path.join(ROOT, "tests"), str(at / "waiting.cpp"), "-o", str(at / "waiting.so")], check=True)
    return str(at / "waiting.so")


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c[0])
def test_other_threads_run_while_a_call_launches(runtime, call):
    r = subprocess.run([sys.executable, "-c", _MAIN, runtime, ROOT], input=json.dumps(call), capture_output=True, text=True, cwd=ROOT, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["0"]
