"""A stream belongs to a device: include/kv.h's calls on the stream of another device than the current one, whose tensors they check, are refused.
No GPU is needed, nothing is launched."""
import importlib

import pytest

from tests.test_kv_abi import P, ROPE, A  # noqa: F401  (A: the fixture)


class Stream:
    """What the calls look at of a torch stream."""

    def __init__(self, device):
        self.cuda_stream, self.device_index = 0, device


CALLS = [("rope_qkv", dict(ROPE, q=P, k=P, v=P, B=1, Hq=2, Hkv=1, N=0, d=64)),
         ("rope_qkv_bwd", dict(ROPE, dq=P, dk=P, dv=P, dqkv=P, dld=256, dq_weight=P, dk_weight=P, workspace=P, B=1, Hq=2, Hkv=1, N=0, d=64)),
         ("kv_append", dict(ROPE, seq=P, pages=P, q=P, k_cache=P, v_cache=P, T=0, S=4, Hq=2, Hkv=1, d=64, W=2, page_size=16, num_pages=9, dtype=0)),
         ("kv_decode", dict(q=P, k_cache=P, v_cache=P, pages=P, lens=P, o=P, lse=P, workspace=P, B=0, Hq=4, Hkv=2, d=64, W=2, page_size=16, num_pages=9, scale=0.1, dtype=0))]


@pytest.mark.parametrize("name,kw", CALLS, ids=lambda x: x if isinstance(x, str) else "")
def test_streams_of_another_device_are_refused(A, monkeypatch, name, kw):  # noqa: F811
    kv = importlib.import_module("paper_2605_10905_amd.kv")
    monkeypatch.setattr(kv, "_device", lambda: 1)
    with pytest.raises(ValueError, match="the stream is on device 0, the current one is 1"):
        getattr(kv, name)(**kw, stream=Stream(0), check=False)
    # its own, and an address (whose device nobody knows), go on to the check of the sizes
    assert getattr(kv, name)(**kw, stream=Stream(1), check=False) == 2 and getattr(kv, name)(**kw, stream=0, check=False) == 2
