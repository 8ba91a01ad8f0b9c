"""Which launches the calls of include/kv.h make, as its documentation says them, and sizes at the ends of what is accepted; behind a runtime
that launches nothing."""
import pytest

from tests.kv_long_cases import APPEND, ROPE
from tests.test_kv_abi import P, _all_calls, _routes

PAGED = dict(seq=P, pages=P, q=P, k_cache=P, v_cache=P, W=2, page_size=16, num_pages=9)


def _rows(Hq, Hkv, d, norm=True):
    w = P if norm else None
    return dict(qkv=P, ld=(Hq + 2 * Hkv) * d, q_weight=w, k_weight=w, eps=1e-5, table=P, npos=8, rot=d, interleaved=0, pos=P)


def test_as_many_kernels_as_documented(tmp_path):
    calls = _all_calls()
    got, _ = _routes(tmp_path, calls)
    for (name, kw), (st, launches) in zip(calls, got):
        want = {"rope_qkv": 1, "rope_qkv_bwd": 2 if kw.get("q_weight") else 1, "kv_append": 1, "kv_decode": 2}[name]
        assert st == 0 and len(launches) == want, (name, kw, launches)


def test_the_long_cases_take_more_than_one_step_of_a_wave(tmp_path):
    """What tests/test_gpu_kv_long.py runs: by one step of a wave each, the rows would need more workgroups of four waves."""
    calls, fewer = [], []
    for c in ROPE:
        B, N, Hq, Hkv, d = c[:5]
        calls.append(("rope_qkv", dict(_rows(Hq, Hkv, d), q=P, k=P, v=P, B=B, Hq=Hq, Hkv=Hkv, N=N, d=d, npos=2 ** 20)))
        steps = -(-B * N * (Hq + 2 * Hkv) // (1024 // d))
        fewer.append(-(-steps // 4) // 2)
        assert steps > 4096 + 4096 // 4  # (the backward: more than one task of each wave of 1024 workgroups of four)
    for c in APPEND:
        T, Hq, Hkv, d = c[:4]
        calls += [("kv_append", dict(_rows(Hq, Hkv, d), **PAGED, T=T, S=T, Hq=Hq, Hkv=Hkv, d=d, dtype=t)) for t in (0, 1)]
        groups = -(-(Hq + 2 * Hkv) // (1024 // d))
        fewer += [-(-T * groups // 4) - 1] * 2
        assert groups > 1
    got, _ = _routes(tmp_path, calls)
    for (name, kw), (st, launches), most in zip(calls, got, fewer):
        assert st == 0 and launches[0][1] <= most, (name, kw, launches, most)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (64, 8), (1021, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_the_most_rows_that_are_accepted(tmp_path, Hq, Hkv, d):
    H = Hq + 2 * Hkv
    most = (2 ** 31 - 1024) // H
    rows = _rows(Hq, Hkv, d)
    calls = [("kv_append", dict(rows, **PAGED, T=T, S=2 ** 31 - 1, Hq=Hq, Hkv=Hkv, d=d, dtype=t)) for T in (most, most + 1) for t in (0, 1)]
    calls += [("rope_qkv", dict(rows, q=P, k=P, v=P, B=1, Hq=Hq, Hkv=Hkv, N=N, d=d)) for N in (most, most + 1)]
    calls += [("rope_qkv_bwd", dict(rows, dq=P, dk=P, dv=P, dqkv=P, dld=H * d, dq_weight=P, dk_weight=P, workspace=P, B=1, Hq=Hq, Hkv=Hkv, N=N, d=d)) for N in (most, most + 1)]
    got, _ = _routes(tmp_path, calls)
    for (name, kw), (st, launches) in zip(calls, got):
        if kw.get("T", kw.get("N")) > most:
            assert st == 4 and not launches, (name, st)
        else:
            assert st == 0 and launches and all(0 < g and g * t < 2 ** 32 for _, g, t in launches), (name, st, launches)
