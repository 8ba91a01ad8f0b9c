"""Arguments that include/kv.h says are not used are not looked at by the binding either.  No GPU is needed: every call ends at a later check."""
import pytest
import torch

from tests.test_kv_abi import P, ROPE, A  # noqa: F401  (A: the fixture)

SHAPE = 2


def _bwd(A, **kw):
    a = dict(ROPE, dq=P, dk=P, dv=P, dqkv=P, dld=4 * 64 - 8, dq_weight=P, dk_weight=P, workspace=P, B=1, Hq=2, Hkv=1, N=8, d=64)  # (dld: too small)
    a.update(kw)
    return A.rope_qkv_bwd(**a, stream=0, check=False)


SMALL = torch.zeros(3)


@pytest.mark.parametrize("kw", [dict(workspace=SMALL), dict(dq_weight=SMALL, dk_weight=SMALL), dict(workspace=SMALL.bfloat16()), dict(qkv=torch.zeros(3, dtype=torch.bfloat16)),
                                dict(qkv=torch.zeros(3, dtype=torch.bfloat16), ld=-8)], ids=lambda kw: "-".join(kw))
def test_without_weights_the_backward_looks_at_no_rows_and_sums(A, kw):  # noqa: F811
    assert _bwd(A, q_weight=None, k_weight=None, **kw) == SHAPE
    with pytest.raises(ValueError):
        _bwd(A, **kw)
    with pytest.raises(ValueError):  # (one weight without the other is refused by the library, which is not reached)
        _bwd(A, q_weight=None, **kw)
