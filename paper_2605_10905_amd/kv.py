"""Python binding of include/kv.h: same names, argument marshalling only.

Beside device addresses the calls take torch tensors, whose type, device, layout and size are checked: a mistake there would
otherwise be read as other numbers, or past the end, by the GPU.  The checks are compiled (csrc/kv_call.cpp)."""
from __future__ import annotations

import ctypes as C
import os

import torch

from .binding import HERE, AttnError
from .binding import _stream as _stream_of
from .build import CALL_KV

lib_path = os.path.join(HERE, "libkv_mi355x.so")
_BUILD = "build it first with `python -m paper_2605_10905_amd.build` (there is no fallback path)"


def _load():
    for path in (lib_path, CALL_KV):
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: {_BUILD}")
    return C.CDLL(lib_path)


lib = _load()
from . import _kv_call as _call  # noqa: E402  (after the library that it calls)

if _call.built_for_torch != torch.__version__:  # (it reads tensors by their layout in memory)
    raise ImportError(f"{CALL_KV} was built for torch {_call.built_for_torch}, this is {torch.__version__}: {_BUILD}")

_i, _ll = C.c_int, C.c_longlong
lib.rope_qkv_bwd_workspace_bytes.argtypes = [_i] * 5
lib.rope_qkv_bwd_workspace_bytes.restype = _ll
lib.kv_decode_workspace_bytes.argtypes = [_i] * 4
lib.kv_decode_workspace_bytes.restype = _ll


def _device():
    """The current device; -1 (no tensor's) where there is none."""
    try:
        return torch._C._cuda_getDevice()  # (torch.cuda.current_device without 150 ns of Python)
    except AttributeError:
        return torch.cuda.current_device()
    except RuntimeError:
        return -1


def _stream(stream, device):
    if stream is None:
        try:
            return torch._C._cuda_getCurrentRawStream(device)  # (the handle alone, as the other calls take it)
        except (AttributeError, RuntimeError):
            pass
    elif getattr(stream, "device_index", device) != device:
        raise ValueError(f"the stream is on device {stream.device_index}, the current one is {device}")
    return _stream_of(stream) or 0


def _done(st, check, call):
    if st != 0 and check:
        raise AttnError(st, call)
    return st


def rope_qkv(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, q, k, v, B, Hq, Hkv, N, d, stream=None, check=True):
    D = _device()
    return _done(_call.rope_qkv(D, _stream(stream, D), qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, q, k, v, B, Hq, Hkv, N, d),
                 check, "rope_qkv")


def rope_qkv_bwd_workspace_bytes(B: int, Hq: int, Hkv: int, N: int, d: int) -> int:
    return lib.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d)


def rope_qkv_bwd(dq, dk, dv, qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, dqkv, dld, dq_weight, dk_weight, workspace,
                 B, Hq, Hkv, N, d, stream=None, check=True):
    D = _device()
    return _done(_call.rope_qkv_bwd(D, _stream(stream, D), dq, dk, dv, qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, dqkv, dld,
                                    dq_weight, dk_weight, workspace, B, Hq, Hkv, N, d), check, "rope_qkv_bwd")


def kv_append(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, seq, pages, q, k_cache, v_cache, T, S, Hq, Hkv, d,
              W, page_size, num_pages, dtype, k_descale=1.0, v_descale=1.0, stream=None, check=True):
    D = _device()
    return _done(_call.kv_append(D, _stream(stream, D), qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, seq, pages, q, k_cache,
                                 v_cache, T, S, Hq, Hkv, d, W, page_size, num_pages, dtype, k_descale, v_descale), check, "kv_append")


def kv_decode_workspace_bytes(B: int, Hq: int, Hkv: int, d: int) -> int:
    return lib.kv_decode_workspace_bytes(B, Hq, Hkv, d)


def kv_decode(q, k_cache, v_cache, pages, lens, o, lse, workspace, B, Hq, Hkv, d, W, page_size, num_pages, scale, dtype, k_descale=1.0,
              v_descale=1.0, stream=None, check=True):
    D = _device()
    return _done(_call.kv_decode(D, _stream(stream, D), q, k_cache, v_cache, pages, lens, o, lse, workspace, B, Hq, Hkv, d, W, page_size, num_pages,
                                 scale, dtype, k_descale, v_descale), check, "kv_decode")
