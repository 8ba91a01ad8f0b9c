"""Numbers with which include/kv.h's calls could not compute are refused, others are not: no GPU is needed, nothing is launched."""
import pytest

from tests.test_kv_abi import P, ROPE, A, _routes  # noqa: F401  (A: the fixture)

UNSUPPORTED = 4
INF = float("inf")


def _decode(A, **kw):
    a = dict(q=P, k_cache=P, v_cache=P, pages=P, lens=P, o=P, lse=P, workspace=P, B=2, Hq=4, Hkv=2, d=64, W=2, page_size=16, num_pages=9, scale=0.1, dtype=1)
    a.update(kw)
    return A.kv_decode(**a, stream=0, check=False)


def _append(A, **kw):
    a = dict(ROPE, seq=P, pages=P, q=P, k_cache=P, v_cache=P, T=4, S=4, Hq=2, Hkv=1, d=64, W=2, page_size=16, num_pages=9, dtype=1)
    a.update(kw)
    return A.kv_append(**a, stream=0, check=False)


# scale * log2(e) * k_descale is what scores are multiplied by: as zero or infinity it would make NaN of hidden keys' -inf, or of the largest score's 0
@pytest.mark.parametrize("kw", [dict(scale=1e-25, k_descale=1e-25), dict(scale=1e20, k_descale=1e30), dict(scale=INF), dict(scale=INF, dtype=0), dict(scale=1e-40, dtype=0),
                                dict(scale=3e38, dtype=0), dict(k_descale=INF), dict(v_descale=INF), dict(k_descale=1e-40), dict(v_descale=2.0 ** -97)], ids=str)
def test_scales_that_leave_the_range_of_float32_are_refused(A, kw):  # noqa: F811
    assert _decode(A, **kw) == UNSUPPORTED


@pytest.mark.parametrize("kw", [dict(k_descale=INF), dict(v_descale=INF), dict(k_descale=2.0 ** -97), dict(v_descale=1e-40)], ids=str)
def test_descales_that_leave_the_range_of_float32_are_refused(A, kw):  # noqa: F811
    assert _append(A, **kw) == UNSUPPORTED


def test_what_can_be_computed_is_taken(tmp_path):
    """The ends of the ranges, and de-scales of a bf16 cache, which are not used.  (Behind a runtime that launches nothing.)"""
    decode = dict(q=P, k_cache=P, v_cache=P, pages=P, lens=P, o=P, lse=P, workspace=P, B=2, Hq=4, Hkv=2, d=64, W=2, page_size=16, num_pages=9, scale=0.1, dtype=1)
    append = dict(ROPE, seq=P, pages=P, q=P, k_cache=P, v_cache=P, T=4, S=4, Hq=2, Hkv=1, d=64, W=2, page_size=16, num_pages=9, dtype=1)
    low, high = 2.0 ** -96, 3.4e38
    calls = [("kv_decode", dict(decode, **kw)) for kw in (dict(k_descale=low, v_descale=low), dict(scale=1e-6, k_descale=high, v_descale=high), dict(scale=2.3e38, dtype=0),
                                                          dict(scale=1e-37, dtype=0), dict(dtype=0, k_descale=0.0, v_descale=1e39), dict(dtype=0, k_descale=-1.0, v_descale=0.0))]
    calls += [("kv_append", dict(append, **kw)) for kw in (dict(k_descale=low, v_descale=high), dict(dtype=0, k_descale=0.0, v_descale=1e39))]
    got, _ = _routes(tmp_path, calls)
    for (name, kw), (st, launches) in zip(calls, got):
        assert st == 0 and len(launches) == (2 if name == "kv_decode" else 1), (name, kw, st)


def test_workspace_sizes_of_sizes_that_no_call_takes(A):  # noqa: F811
    """They do not wrap around: enough, or as much as the largest call needs."""
    big = 2 ** 31 - 1
    assert A.rope_qkv_bwd_workspace_bytes(big, big, big, big, 128) == A.rope_qkv_bwd_workspace_bytes(64, 64, 64, 1 << 20, 128)
    assert A.rope_qkv_bwd_workspace_bytes(1, 1, 1, 1, big) == 2 * 4 * big
    for shape in ((1, 1, 1, 2 ** 27), (1, 64, 1, 2 ** 26), (big, 64, 1, 128), (big, big, 1, 64), (big, big, big, 64)):
        B, Hq, Hkv, d = shape
        assert A.kv_decode_workspace_bytes(*shape) >= 2 * 1024 * min(Hq // Hkv, 16) * d * 4, shape
