"""The boundary of include/kv.h without a GPU: symbols, refusals, the binding's checks of tensors, and which kernels a call
launches (behind a runtime that only writes launches down, launch_recorder.cpp)."""
import ctypes
import importlib
import json
import os
import re
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def A():
    import paper_2605_10905_amd as A

    return A


def test_every_declared_symbol_is_exported_and_reachable(A):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "kv.h")).read(), flags=re.S)
    names = set(re.findall(r"\b((?:rope|kv)_[a-z0-9_]+)\s*\(", text))
    assert {"rope_qkv", "rope_qkv_bwd", "kv_append", "kv_decode"} <= names
    lib = importlib.import_module("paper_2605_10905_amd.kv").lib
    for n in names:
        assert hasattr(lib, n) and callable(getattr(A, n)) and n in dir(A)


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "kv.h"\nint main(void){return (int)kv_decode_workspace_bytes(0, 0, 0, 0);}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "t.o")], check=True)


ROPE = dict(qkv=P, ld=4 * 64, q_weight=P, k_weight=P, eps=1e-5, table=P, npos=8, rot=64, interleaved=0, pos=P)


def _rope(A, **kw):
    a = dict(ROPE, q=P, k=P, v=P, B=1, Hq=2, Hkv=1, N=8, d=64, **{})
    a.update(kw)
    return A.rope_qkv(**a, stream=0, check=False)


def _bwd(A, **kw):
    a = dict(ROPE, dq=P, dk=P, dv=P, dqkv=P, dld=4 * 64, dq_weight=P, dk_weight=P, workspace=P, B=1, Hq=2, Hkv=1, N=8, d=64)
    a.update(kw)
    return A.rope_qkv_bwd(**a, stream=0, check=False)


def _append(A, **kw):
    a = dict(ROPE, seq=P, pages=P, q=P, k_cache=P, v_cache=P, T=4, S=4, Hq=2, Hkv=1, d=64, W=2, page_size=16, num_pages=9, dtype=0)
    a.update(kw)
    return A.kv_append(**a, stream=0, check=False)


def _decode(A, **kw):
    a = dict(q=P, k_cache=P, v_cache=P, pages=P, lens=P, o=P, lse=P, workspace=P, B=2, Hq=4, Hkv=2, d=64, W=2, page_size=16, num_pages=9, scale=0.1, dtype=0)
    a.update(kw)
    return A.kv_decode(**a, stream=0, check=False)


@pytest.mark.parametrize("call", [_rope, _bwd, _append])
def test_rows_are_checked(A, call):
    size = "T" if call is _append else "N"
    missing = dict(_rope=("qkv", "q_weight", "k_weight", "table", "q", "k", "v"), _append=("qkv", "k_weight", "table", "pos", "pages", "q", "k_cache", "v_cache"),
                   _bwd=("qkv", "q_weight", "table", "dq", "dk", "dv", "dqkv", "dq_weight", "dk_weight", "workspace"))[call.__name__]
    for name in missing:
        assert call(A, **{name: None}) == 1, name
    for kw in ({size: 0}, {size: -3}, dict(Hq=3, Hkv=2), dict(Hkv=0), dict(ld=4 * 64 - 8), dict(ld=4 * 64 + 4), dict(rot=-16), dict(rot=80), dict(npos=0), dict(qkv=P + 8),
               dict(table=P + 4), dict(k_weight=P + 2), dict(pos=P + 2), dict(d=0)):
        assert call(A, **kw) == 2, kw
    for kw in (dict(d=32, rot=32), dict(d=96, ld=4 * 96), dict(d=256, ld=4 * 256), dict(rot=24), dict(eps=-1.0), dict(eps=float("nan")), {size: 2 ** 30}, {size: (2 ** 31 - 1024) // 4 + 1}):
        assert call(A, **kw) == 4, kw


def test_the_rest_is_checked(A):
    assert _rope(A, N=9, pos=None) == 2 and _rope(A, B=0) == 2 and _rope(A, v=P + 4) == 2      # more tokens than the table has positions
    assert _bwd(A, N=9, pos=None) == 2 and _bwd(A, dld=4 * 64 - 8) == 2 and _bwd(A, workspace=P + 4) == 2 and _bwd(A, dqkv=P + 2) == 2
    assert _append(A, seq=None, T=5) == 2 and _append(A, W=0) == 2 and _append(A, num_pages=0) == 2 and _append(A, S=0) == 2 and _append(A, seq=P + 1) == 2
    assert _append(A, dtype=7) == 3 and _decode(A, dtype=-1) == 3
    for size in (8, 24, 2048, 17):
        assert _append(A, page_size=size) == 4 and _decode(A, page_size=size) == 4
    for bad in (0.0, -1.0, float("nan")):
        assert _append(A, dtype=1, k_descale=bad) == 4 and _append(A, dtype=1, v_descale=bad) == 4
        assert _decode(A, dtype=1, k_descale=bad) == 4 and _decode(A, dtype=1, v_descale=bad) == 4 and _decode(A, scale=bad) == 4
    for name in ("q", "k_cache", "v_cache", "pages", "lens", "o", "lse", "workspace"):
        assert _decode(A, **{name: None}) == 1, name
        assert _decode(A, **{name: P + 2}) == 2, name
    assert _decode(A, B=0) == 2 and _decode(A, Hq=5) == 2 and _decode(A, Hkv=0) == 2 and _decode(A, d=80) == 4 and _decode(A, page_size=0) == 2
    assert _decode(A, W=2 ** 28, page_size=16) == 4 and _decode(A, B=2 ** 23, Hq=4) == 4
    with pytest.raises(A.AttnError):
        A.kv_decode(None, P, P, P, P, P, P, P, 1, 1, 1, 64, 1, 16, 1, 1.0, 0, stream=0)


def test_workspace_sizes(A):
    assert A.rope_qkv_bwd_workspace_bytes(0, 1, 1, 1, 64) == 0 and A.rope_qkv_bwd_workspace_bytes(1, 1, 1, 1, 64) == 2 * 64 * 4
    big = A.rope_qkv_bwd_workspace_bytes(64, 64, 64, 1 << 20, 128)
    assert 0 < big <= 4 << 20 and big == A.rope_qkv_bwd_workspace_bytes(64, 64, 64, 1 << 21, 128)
    assert A.kv_decode_workspace_bytes(0, 1, 1, 64) == 0 and A.kv_decode_workspace_bytes(1, 3, 2, 64) == 0
    for shape in ((1, 1, 1, 64), (64, 64, 8, 128), (3, 130, 2, 128)):
        n = A.kv_decode_workspace_bytes(*shape)
        assert n > 0 and n % 16 == 0


def test_tensors_that_the_gpu_could_not_read_are_refused(A):
    """Other types, CPU tensors, strides and too few elements are errors of the binding, before the library is called."""
    bf, i32 = torch.zeros(4096, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.int32)
    f32 = torch.zeros(A.kv_decode_workspace_bytes(2, 4, 2, 64) // 4)
    for kw, text in ((dict(q=bf.float()), "q is Float, not BFloat16"), (dict(q=bf), "q is not on a GPU"), (dict(lens=i32.long()), "lens is Long, not Int"),
                     (dict(lens=i32), "not on a GPU"), (dict(k_cache=bf, dtype=1), "k_cache is BFloat16, not Byte"), (dict(workspace=bf), "not Float"),
                     (dict(v_cache=bf.view(torch.uint8)), "v_cache is Byte, not BFloat16"), (dict(workspace=f32), "workspace is not on a GPU"),
                     (dict(workspace=f32[1:]), "elements"), (dict(pages=i32[:3]), "pages has 3 elements, 4 are needed"), (dict(o=bf.view(64, 64).t()), "o must be contiguous")):
        with pytest.raises(ValueError, match=text):
            _decode(A, **kw)
    for call, kw in ((_rope, dict(qkv=bf)), (_rope, dict(pos=i32.float())), (_bwd, dict(dqkv=bf)), (_append, dict(seq=i32)), (_append, dict(v_cache=i32))):
        with pytest.raises(ValueError):
            call(A, **kw)


def test_rows_of_a_wider_buffer_are_checked(A):
    """Views whose rows are `ld` apart are taken (the next check, of the device, is the one that fails here), others are not."""
    x = torch.zeros(9, 320, dtype=torch.bfloat16)
    for t, ld, B, N in ((x[:8, :256], 320, 1, 8), (x[:, 64:], 320, 1, 9), (x.view(3, 3, 320)[:, :, 8:264], 320, 3, 3), (x.view(-1), 320, 3, 3), (x, 256, 1, 8), (x[:1, :256], 320, 1, 1),
                        (x[1:2], 320, 1, 1), (x[4:, :300], 320, 5, 1)):
        with pytest.raises(ValueError, match="qkv is not on a GPU"):
            _rope(A, qkv=t, ld=ld, B=B, N=N, npos=99)
        with pytest.raises(ValueError, match="dqkv is not on a GPU"):
            _bwd(A, dqkv=t, dld=ld, B=B, N=N, npos=99)
    for t, ld, B, N in ((x, 336, 1, 9), (x, 320, 2, 5), (x[:, :200], 320, 1, 9), (x[::2, :256], 320, 1, 5), (x[:, :256], 256, 1, 9), (x[:, ::1].t(), 8, 1, 320),
                        (x.view(3, 3, 320)[:, :2], 320, 3, 2), (x.view(3, 3, 320)[::2], 320, 2, 3), (x[:1, :256], 320, 1, 2), (x[:, ::5], 320, 1, 9)):
        with pytest.raises(ValueError, match="does not hold"):
            _rope(A, qkv=t, ld=ld, B=B, N=N, npos=999)


def test_arguments_that_are_no_numbers_or_tensors(A):
    import numpy as np

    with pytest.raises(TypeError):
        _decode(A, q=[1.0])
    with pytest.raises(TypeError):
        _decode(A, B="2")
    with pytest.raises(TypeError):
        _decode(A, scale=None)
    with pytest.raises(OverflowError):
        _decode(A, W=2 ** 31)
    with pytest.raises(OverflowError):
        _rope(A, ld=2 ** 63)
    assert _decode(A, B=np.int64(0)) == 2 and _decode(A, scale=np.float32(-1)) == 4 and _rope(A, interleaved=True, N=0) == 2
    with pytest.raises(TypeError):
        importlib.import_module("paper_2605_10905_amd.kv")._call.kv_decode(0, 0, 1, 2)


_MAIN = """
import ctypes, json, sys
import torch  # (its own kernels are not ours to write down)
rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
rec.recorder_take.restype = rec.recorder_kernels.restype = ctypes.c_char_p
sys.path.insert(0, sys.argv[2])
import importlib
importlib.import_module("paper_2605_10905_amd.binding")
before = set(rec.recorder_kernels().decode().splitlines())
kv = importlib.import_module("paper_2605_10905_amd.kv")
own = [x.split("\\t")[0] for x in rec.recorder_kernels().decode().splitlines() if x not in before]
calls = []
for name, kw in json.load(sys.stdin):
    st = getattr(kv, name)(**kw, stream=0, check=False)
    calls.append((st, [x.split("\\t") for x in rec.recorder_take().decode().splitlines()]))
json.dump(dict(calls=calls, kernels=own), sys.stdout)
"""


def _routes(tmp_path, calls):
    lib = tmp_path / "recorder.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "launch_recorder.cpp"), "-o", str(lib)], check=True)
    r = subprocess.run([sys.executable, "-c", _MAIN, str(lib), ROOT], input=json.dumps(calls), capture_output=True, text=True, cwd=ROOT, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    got = json.loads(r.stdout)
    short = lambda n: re.sub(r"\(.*", "", n.replace("(anonymous namespace)::", "").replace("void ", ""))
    return [(st, [(short(n), int(g), int(t)) for n, g, t in launches]) for st, launches in got["calls"]], {short(n) for n in got["kernels"]}


def _all_calls():
    calls = []
    for d in (64, 128):
        for norm in (False, True):
            w = P if norm else None
            rope = dict(ROPE, q_weight=w, k_weight=w, ld=16 * d)
            for Hq, Hkv in ((12, 2), (5, 1)):  # (16 heads are whole steps of a wave, 7 are not)
                size = dict(B=2, Hq=Hq, Hkv=Hkv, N=5, d=d)
                calls += [("rope_qkv", dict(rope, q=P, k=P, v=P, **size)),
                          ("rope_qkv_bwd", dict(rope, dq=P, dk=P, dv=P, dqkv=P, dld=16 * d, dq_weight=w, dk_weight=w, workspace=w, **size))]
            calls += [("kv_append", dict(rope, seq=P, pages=P, q=P, k_cache=P, v_cache=P, T=4, S=4, Hq=2, Hkv=1, d=d, W=2, page_size=16, num_pages=9, dtype=t)) for t in (0, 1)]
        # few and many (sequence, key head) pairs: 2, 100 and 200 of them, more with many heads to one
        calls += [("kv_decode", dict(q=P, k_cache=P, v_cache=P, pages=P, lens=P, o=P, lse=P, workspace=P, B=B, Hq=G, Hkv=1, d=d, W=2, page_size=16, num_pages=9,
                                     scale=0.1, dtype=t)) for t in (0, 1) for G in (1, 5, 16, 17, 32, 33, 65) for B in (2, 100, 200)]
    return calls


def test_every_kernel_is_launched_by_some_call(tmp_path):
    """All of these kinds of calls (head dimension, norm, cache type, heads that share a key head) are run by tests/test_gpu_kv.py."""
    calls = _all_calls()
    got, kernels = _routes(tmp_path, calls)
    assert all(st == 0 for st, _ in got)
    assert kernels and kernels == {n for _, launches in got for n, _, _ in launches}
    for (name, kw), (_, launches) in zip(calls, got):
        assert len(launches) == (2 if name == "rope_qkv_bwd" and kw["q_weight"] else len(launches))
        assert all(g * t < 2 ** 32 for _, g, t in launches)


def test_the_largest_sizes_fit_a_launch(tmp_path):
    big = [("rope_qkv", dict(ROPE, ld=192, q=P, k=P, v=P, B=1, Hq=1, Hkv=1, N=700_000_000, d=64, npos=1)),
           ("rope_qkv_bwd", dict(ROPE, ld=192, dq=P, dk=P, dv=P, dqkv=P, dld=192, dq_weight=P, dk_weight=P, workspace=P, B=1, Hq=1, Hkv=1, N=700_000_000, d=64)),
           ("kv_decode", dict(q=P, k_cache=P, v_cache=P, pages=P, lens=P, o=P, lse=P, workspace=P, B=2 ** 22 - 1, Hq=4, Hkv=4, d=64, W=2 ** 20, page_size=1024, num_pages=2 ** 30,
                              scale=0.1, dtype=0))]
    got, _ = _routes(tmp_path, big)
    for (name, _), (st, launches) in zip(big, got):
        assert st == 0 and launches and all(0 < g and g * t < 2 ** 32 for _, g, t in launches), (name, st, launches)
