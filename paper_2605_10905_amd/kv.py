"""ctypes binding of include/kv.h: same names, argument marshalling only.

Beside device addresses the calls take torch tensors, whose type, device, layout and size are checked: a mistake there would
otherwise be read as other numbers, or past the end, by the GPU."""
from __future__ import annotations

import ctypes as C
import os

import torch

from .binding import HERE, AttnError
from .binding import _stream as _stream_of

lib_path = os.path.join(HERE, "libkv_mi355x.so")


def _load():
    if not os.path.exists(lib_path):
        raise ImportError(
            f"{lib_path} is missing: build it first with `python -m paper_2605_10905_amd.build` "
            "(there is no fallback path)")
    return C.CDLL(lib_path)


lib = _load()

_vp, _i, _f, _ll = C.c_void_p, C.c_int, C.c_float, C.c_longlong
_ROPE = [_vp, _ll, _vp, _vp, _f, _vp, _i, _i, _i, _vp]  # qkv .. pos
lib.rope_qkv.argtypes = _ROPE + [_vp] * 3 + [_i] * 5 + [_vp]
lib.rope_qkv.restype = _i
lib.rope_qkv_bwd.argtypes = [_vp] * 3 + _ROPE + [_vp, _ll] + [_vp] * 3 + [_i] * 5 + [_vp]
lib.rope_qkv_bwd.restype = _i
lib.rope_qkv_bwd_workspace_bytes.argtypes = [_i] * 5
lib.rope_qkv_bwd_workspace_bytes.restype = _ll
lib.kv_append.argtypes = _ROPE + [_vp] * 5 + [_i] * 9 + [_f, _f, _vp]
lib.kv_append.restype = _i
lib.kv_decode.argtypes = [_vp] * 8 + [_i] * 7 + [_f, _i, _f, _f, _vp]
lib.kv_decode.restype = _i
lib.kv_decode_workspace_bytes.argtypes = [_i] * 4
lib.kv_decode_workspace_bytes.restype = _ll

_BF16, _F32, _I32, _U8, _E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn


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
    return _stream_of(stream)


# A small call takes as long as the host takes for it, so a tensor's checks are one expression: 0.25 us each, ten of them in kv_append.
def _ptr(t, dtype, least, device, name):
    """Address of a tensor of at least `least` elements (what the call reads or writes), or of what is an address already."""
    try:
        if t.dtype is dtype and t.get_device() == device and t.is_contiguous() and t.numel() >= least and device >= 0:
            return t.data_ptr()
    except AttributeError:
        if t is None or isinstance(t, int):
            return t
        raise TypeError(f"{name} is {type(t).__name__}, not a tensor or an address") from None
    _refuse_other(t, dtype, device, name)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} has {t.numel()} elements, {least} are needed")


def _refuse_other(t, dtype, device, name):
    if t.dtype is not dtype:
        raise ValueError(f"{name} is {t.dtype}, not {dtype}")
    if t.get_device() < 0:
        raise ValueError(f"{name} is not on a GPU")
    if t.get_device() != device:
        raise ValueError(f"{name} is on device {t.get_device()}, the current one is {device}")


def _rows(t, ld, rows, width, device, name):
    """Address of `rows` rows of `width` bf16 features, `ld` elements apart."""
    try:
        if t.dtype is _BF16 and t.get_device() == device and t.is_contiguous() and t.numel() >= (rows - 1) * ld + width and device >= 0:
            return t.data_ptr()  # (a dense buffer may be given in any shape)
    except AttributeError:
        if t is None or isinstance(t, int):
            return t
        raise TypeError(f"{name} is {type(t).__name__}, not a tensor or an address") from None
    _refuse_other(t, _BF16, device, name)
    shape, stride = t.shape, t.stride()
    ok = not t.is_contiguous() and shape[-1] >= width and stride[-1] == 1
    step, count = ld, 1
    for n, s in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        ok = ok and (n == 1 or s == step)
        step *= n
        count *= n
    if not ok or count < rows:
        raise ValueError(f"{name} (shape {tuple(shape)}, strides {tuple(stride)}) does not hold {rows} rows of {width}, {ld} apart")
    return t.data_ptr()


def _cache(t, dtype, least, device, name):
    """e4m3 caches are bytes, or torch's type of them."""
    kind = _BF16 if dtype != 1 else _E4M3 if getattr(t, "dtype", None) is _E4M3 else _U8
    return _ptr(t, kind, least, device, name)


def _done(st, check, call):
    if check and st != 0:
        raise AttnError(st, call)
    return st


def rope_qkv(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, q, k, v, B, Hq, Hkv, N, d, stream=None, check=True):
    D, T = _device(), B * N
    nk = T * Hkv * d
    st = lib.rope_qkv(_rows(qkv, ld, T, (Hq + 2 * Hkv) * d, D, "qkv"), ld, _ptr(q_weight, _BF16, d, D, "q_weight"), _ptr(k_weight, _BF16, d, D, "k_weight"), eps,
                      _ptr(table, _F32, npos * rot, D, "table"), npos, rot, 1 if interleaved else 0, _ptr(pos, _I32, T, D, "pos"),
                      _ptr(q, _BF16, T * Hq * d, D, "q"), _ptr(k, _BF16, nk, D, "k"), _ptr(v, _BF16, nk, D, "v"), B, Hq, Hkv, N, d, _stream(stream, D))
    return _done(st, check, "rope_qkv")


def rope_qkv_bwd_workspace_bytes(B: int, Hq: int, Hkv: int, N: int, d: int) -> int:
    return lib.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d)


def rope_qkv_bwd(dq, dk, dv, qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, dqkv, dld, dq_weight, dk_weight, workspace,
                 B, Hq, Hkv, N, d, stream=None, check=True):
    D, T, width = _device(), B * N, (Hq + 2 * Hkv) * d
    nk, need = T * Hkv * d, lib.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4
    st = lib.rope_qkv_bwd(_ptr(dq, _BF16, T * Hq * d, D, "dq"), _ptr(dk, _BF16, nk, D, "dk"), _ptr(dv, _BF16, nk, D, "dv"), _rows(qkv, ld, T, width, D, "qkv"), ld,
                          _ptr(q_weight, _BF16, d, D, "q_weight"), _ptr(k_weight, _BF16, d, D, "k_weight"), eps, _ptr(table, _F32, npos * rot, D, "table"), npos, rot,
                          1 if interleaved else 0, _ptr(pos, _I32, T, D, "pos"), _rows(dqkv, dld, T, width, D, "dqkv"), dld, _ptr(dq_weight, _F32, d, D, "dq_weight"),
                          _ptr(dk_weight, _F32, d, D, "dk_weight"), _ptr(workspace, _F32, need, D, "workspace"), B, Hq, Hkv, N, d, _stream(stream, D))
    return _done(st, check, "rope_qkv_bwd")


def kv_append(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, seq, pages, q, k_cache, v_cache, T, S, Hq, Hkv, d,
              W, page_size, num_pages, dtype, k_descale=1.0, v_descale=1.0, stream=None, check=True):
    D, held = _device(), num_pages * Hkv * page_size * d
    st = lib.kv_append(_rows(qkv, ld, T, (Hq + 2 * Hkv) * d, D, "qkv"), ld, _ptr(q_weight, _BF16, d, D, "q_weight"), _ptr(k_weight, _BF16, d, D, "k_weight"), eps,
                       _ptr(table, _F32, npos * rot, D, "table"), npos, rot, 1 if interleaved else 0, _ptr(pos, _I32, T, D, "pos"), _ptr(seq, _I32, T, D, "seq"),
                       _ptr(pages, _I32, S * W, D, "pages"), _ptr(q, _BF16, T * Hq * d, D, "q"), _cache(k_cache, dtype, held, D, "k_cache"),
                       _cache(v_cache, dtype, held, D, "v_cache"), T, S, Hq, Hkv, d, W, page_size, num_pages, dtype, k_descale, v_descale, _stream(stream, D))
    return _done(st, check, "kv_append")


def kv_decode_workspace_bytes(B: int, Hq: int, Hkv: int, d: int) -> int:
    return lib.kv_decode_workspace_bytes(B, Hq, Hkv, d)


def kv_decode(q, k_cache, v_cache, pages, lens, o, lse, workspace, B, Hq, Hkv, d, W, page_size, num_pages, scale, dtype, k_descale=1.0,
              v_descale=1.0, stream=None, check=True):
    D, held, nq = _device(), num_pages * Hkv * page_size * d, B * Hq * d
    need = lib.kv_decode_workspace_bytes(B, Hq, Hkv, d) // 4
    st = lib.kv_decode(_ptr(q, _BF16, nq, D, "q"), _cache(k_cache, dtype, held, D, "k_cache"), _cache(v_cache, dtype, held, D, "v_cache"),
                       _ptr(pages, _I32, B * W, D, "pages"), _ptr(lens, _I32, B, D, "lens"), _ptr(o, _BF16, nq, D, "o"), _ptr(lse, _F32, B * Hq, D, "lse"),
                       _ptr(workspace, _F32, need, D, "workspace"), B, Hq, Hkv, d, W, page_size, num_pages, scale, dtype, k_descale, v_descale, _stream(stream, D))
    return _done(st, check, "kv_decode")
