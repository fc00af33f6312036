"""Numbers of entries past 32 bits are refused, not taken modulo 2^32.  CPU only
but for the last."""
import os

import pytest
import torch

import paper_2503_12382_amd as reno

pytestmark = pytest.mark.skipif(not os.path.exists(reno.LIB_PATH),
                                reason="libreno.so not built (run __graft_entry__.build())")
BAD = [-1, 0, 129, 2 ** 31, 2 ** 32 + 3, -2 ** 32 + 3]


@pytest.mark.parametrize("k", BAD)
def test_workspace(k):
    with pytest.raises(reno.RenoError) as e:
        reno.head_workspace(10, 64, 256, torch.float32, k, True)
    assert e.value.status == reno.RENO_E_INVALID and str(e.value)


@pytest.mark.gpu
@pytest.mark.parametrize("k", BAD)
def test_top_logits(k):
    with pytest.raises(reno.RenoError) as e:
        reno.top_logits(torch.empty(0, 9, device="cuda"), k)
    assert e.value.status == reno.RENO_E_INVALID and str(e.value)
