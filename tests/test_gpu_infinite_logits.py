"""Logits of +inf: the row's normaliser is +inf, as its definition gives."""
import math

import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


# rows of 16 lanes, of a block that holds them (64, 256 and 1024 threads), of one that reads them twice
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [3, 40, 255, 1000, 9001, 40000, 140001])
def test_top_logits(V, dt):
    x = torch.randn(9, V, generator=torch.Generator().manual_seed(V)).to(dt)
    x[0, 0] = math.inf
    x[1, V - 1] = math.inf
    x[2, V // 2:] = math.inf
    x[3] = math.inf
    x[4] = -math.inf
    x[4, V // 3] = math.inf
    x[5, 0], x[5, V - 1] = math.inf, math.nan
    x[6] = torch.finfo(dt).max
    x[6, 1] = math.inf
    x[7, ::2] = -math.inf
    say("top logits of +inf", V, dt)
    for off in (0, 1):          # rows that start on 16 bytes, and that do not
        buf = torch.zeros(9, V + 16 - V % 8, dtype=dt, device="cuda")
        buf[:, off:off + V] = x.cuda()
        r = reno.top_logits(buf[:, off:off + V], 2)
        want = torch.logsumexp(x.double(), 1)
        assert want[:5].tolist() == [math.inf] * 5 and want[6] == math.inf
        assert r.lse[:5].tolist() == [math.inf] * 5 and r.lse[6] == math.inf
        assert math.isnan(r.lse[5])
        for i in (7, 8):
            assert abs(float(r.lse[i]) - float(want[i])) < 1e-4 * max(1.0, abs(float(want[i])))
        assert r.index[:2, 0].tolist() == [0, V - 1] and r.value[:2, 0].tolist() == [math.inf] * 2
        assert r.index[4, 0] == V // 3 and r.index[6, 0] == 1
        assert r.index[3].tolist() == [0, 1]
