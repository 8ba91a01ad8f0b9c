"""ctypes binding of include/kv.h: same names, argument marshalling only.

Beside device addresses the calls take torch tensors, whose type, device and layout are checked: a mistake there would
otherwise be read as other numbers, or past the end, by the GPU."""
from __future__ import annotations

import ctypes as C
import os

from .binding import HERE, AttnError, _stream

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


def _types():
    import torch

    # (torch is imported when the first tensor comes: the library itself needs none of it)
    global _BF16, _F32, _I32, _U8
    _BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, (torch.uint8, torch.float8_e4m3fn)
    return torch


_BF16 = _F32 = _I32 = _U8 = None
_KINDS = {"bf16": lambda: (_BF16,), "f32": lambda: (_F32,), "i32": lambda: (_I32,), "e4m3": lambda: _U8}


class _Args:
    """Device pointers of the tensors of one call; all of them on the current device."""

    __slots__ = ("call", "device")

    def __init__(self, call):
        self.call, self.device = call, None

    def _checked(self, t, kind, name):
        if _BF16 is None:
            _types()
        if t.dtype not in _KINDS[kind]():
            raise ValueError(f"{self.call}: {name} is {t.dtype}, not {kind}")
        device = t.get_device()
        if device != self.device:
            if device < 0:
                raise ValueError(f"{self.call}: {name} is not on a GPU")
            import torch

            self.device = torch.cuda.current_device()
            if device != self.device:
                raise ValueError(f"{self.call}: {name} is on device {device}, the current one is {self.device}")
        return t.data_ptr()

    def __call__(self, t, kind, name, least=0):
        """`least`: the number of elements that the call reads or writes."""
        if t is None or isinstance(t, int):
            return t
        ptr = self._checked(t, kind, name)
        if not t.is_contiguous():
            raise ValueError(f"{self.call}: {name} must be contiguous")
        if t.numel() < least:
            raise ValueError(f"{self.call}: {name} has {t.numel()} elements, {least} are needed")
        return ptr

    def rows(self, t, ld, rows, width, name):
        """`rows` rows of `width` features, `ld` elements apart."""
        if t is None or isinstance(t, int):
            return t
        ptr = self._checked(t, "bf16", name)
        shape, stride, step = t.shape, t.stride(), ld
        ok = len(shape) > 0 and (shape[-1] == 1 or stride[-1] == 1)
        if t.is_contiguous():  # (a dense buffer may be given in any shape)
            ok = t.numel() >= (rows - 1) * ld + width
        else:
            count = 1
            for n, s in zip(reversed(shape[:-1]), reversed(stride[:-1])):
                ok = ok and (n == 1 or s == step)
                step *= n
                count *= n
            ok = ok and count >= rows and shape[-1] >= width
        if not ok:
            raise ValueError(f"{self.call}: {name} (shape {tuple(shape)}, strides {tuple(stride)}) does not hold {rows} rows of {width}, {ld} apart")
        return ptr


def _rope_args(a, q_weight, k_weight, table, npos, rot, pos, T, d):
    return (a(q_weight, "bf16", "q_weight", d), a(k_weight, "bf16", "k_weight", d), a(table, "f32", "table", npos * rot), a(pos, "i32", "pos", T))


def _done(st, check, call):
    if check and st != 0:
        raise AttnError(st, call)
    return st


def rope_qkv(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, q, k, v, B, Hq, Hkv, N, d, stream=None, check=True):
    a, T = _Args("rope_qkv"), B * N
    wq, wk, tab, ps = _rope_args(a, q_weight, k_weight, table, npos, rot, pos, T, d)
    st = lib.rope_qkv(a.rows(qkv, ld, T, (Hq + 2 * Hkv) * d, "qkv"), ld, wq, wk, eps, tab, npos, rot, 1 if interleaved else 0, ps,
                      a(q, "bf16", "q", T * Hq * d), a(k, "bf16", "k", T * Hkv * d), a(v, "bf16", "v", T * Hkv * d), B, Hq, Hkv, N, d, _stream(stream))
    return _done(st, check, "rope_qkv")


def rope_qkv_bwd_workspace_bytes(B: int, Hq: int, Hkv: int, N: int, d: int) -> int:
    return lib.rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d)


def rope_qkv_bwd(dq, dk, dv, qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, dqkv, dld, dq_weight, dk_weight, workspace,
                 B, Hq, Hkv, N, d, stream=None, check=True):
    a, T, width = _Args("rope_qkv_bwd"), B * N, (Hq + 2 * Hkv) * d
    wq, wk, tab, ps = _rope_args(a, q_weight, k_weight, table, npos, rot, pos, T, d)
    need = rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) // 4 if q_weight is not None else 0
    st = lib.rope_qkv_bwd(a(dq, "bf16", "dq", T * Hq * d), a(dk, "bf16", "dk", T * Hkv * d), a(dv, "bf16", "dv", T * Hkv * d),
                          a.rows(qkv, ld, T, width, "qkv"), ld, wq, wk, eps, tab, npos, rot, 1 if interleaved else 0, ps,
                          a.rows(dqkv, dld, T, width, "dqkv"), dld, a(dq_weight, "f32", "dq_weight", d), a(dk_weight, "f32", "dk_weight", d),
                          a(workspace, "f32", "workspace", need), B, Hq, Hkv, N, d, _stream(stream))
    return _done(st, check, "rope_qkv_bwd")


def kv_append(qkv, ld, q_weight, k_weight, eps, table, npos, rot, interleaved, pos, seq, pages, q, k_cache, v_cache, T, S, Hq, Hkv, d,
              W, page_size, num_pages, dtype, k_descale=1.0, v_descale=1.0, stream=None, check=True):
    a, held, kind = _Args("kv_append"), num_pages * Hkv * page_size * d, "e4m3" if dtype == 1 else "bf16"
    wq, wk, tab, ps = _rope_args(a, q_weight, k_weight, table, npos, rot, pos, T, d)
    st = lib.kv_append(a.rows(qkv, ld, T, (Hq + 2 * Hkv) * d, "qkv"), ld, wq, wk, eps, tab, npos, rot, 1 if interleaved else 0, ps,
                       a(seq, "i32", "seq", T), a(pages, "i32", "pages", S * W), a(q, "bf16", "q", T * Hq * d),
                       a(k_cache, kind, "k_cache", held), a(v_cache, kind, "v_cache", held), T, S, Hq, Hkv, d, W, page_size, num_pages,
                       dtype, k_descale, v_descale, _stream(stream))
    return _done(st, check, "kv_append")


def kv_decode_workspace_bytes(B: int, Hq: int, Hkv: int, d: int) -> int:
    return lib.kv_decode_workspace_bytes(B, Hq, Hkv, d)


def kv_decode(q, k_cache, v_cache, pages, lens, o, lse, workspace, B, Hq, Hkv, d, W, page_size, num_pages, scale, dtype, k_descale=1.0,
              v_descale=1.0, stream=None, check=True):
    a, held, kind = _Args("kv_decode"), num_pages * Hkv * page_size * d, "e4m3" if dtype == 1 else "bf16"
    st = lib.kv_decode(a(q, "bf16", "q", B * Hq * d), a(k_cache, kind, "k_cache", held), a(v_cache, kind, "v_cache", held),
                       a(pages, "i32", "pages", B * W), a(lens, "i32", "lens", B), a(o, "bf16", "o", B * Hq * d), a(lse, "f32", "lse", B * Hq),
                       a(workspace, "f32", "workspace", lib.kv_decode_workspace_bytes(B, Hq, Hkv, d) // 4), B, Hq, Hkv, d, W, page_size, num_pages,
                       scale, dtype, k_descale, v_descale, _stream(stream))
    return _done(st, check, "kv_decode")
