"""Logits of +inf: the row's normaliser is +inf, as its definition gives, in the
selection of the top logits and in the head's operators."""
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


# narrow fp32, wide, few rows
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V,grad", [(40, 20, 90, False), (40, 20, 90, True), (300, 70, 256, True), (40, 20, 700, True),
                                        (40, 20, 700, False), (3, 40, 700, False), (1, 40, 33000, False),
                                        (300, 300, 1500, True)])
def test_head(N, C, V, grad, dt):
    g = torch.Generator().manual_seed(N + C + V)
    h, w = torch.randn(N, C, generator=g).to(dt), (torch.randn(C, V, generator=g) / math.sqrt(C)).to(dt)
    b = torch.zeros(V).to(dt)
    up = V - 2                                   # the symbol whose logit is +inf in every row
    b[up] = math.inf
    b[0] = -math.inf
    s = torch.randint(1, up, (N,), generator=g).int()
    if N > 1:
        s[0], s[1] = up, -1
    if N > 3:
        s[3] = 0
    say("head logits of +inf", N, C, V, grad, dt)
    r = reno.head_code_length(h.cuda(), w.cuda(), b.cuda(), s.cuda(), grad=grad)
    taken = s >= 0
    assert torch.equal(r.lse.cpu(), torch.where(taken, math.inf, 0.0))
    want = torch.where(s == up, math.nan, torch.where(taken, math.inf, 0.0))   # (lse - z_s) / ln 2
    assert torch.equal(r.bits.cpu().nan_to_num(-1.0, posinf=7.0), want.nan_to_num(-1.0, posinf=7.0))
    if grad and N > 1:
        assert not bool(r.dh[1].any())
    index = torch.stack([s, torch.where(taken, (s + 1) % up, -1), torch.full_like(s, -1)], 1).int()
    index[:, 1] = torch.where(index[:, 1] == 0, 5, index[:, 1])
    r = reno.head_distill(h.cuda(), w.cuda(), b.cuda(), index.cuda(), torch.zeros(N, 3).cuda(), temperature=2.0, grad=grad)
    assert torch.equal(r.lse.cpu(), torch.where(taken, math.inf, 0.0))
    assert torch.equal(r.bits.cpu().nan_to_num(-1.0, posinf=7.0), want.nan_to_num(-1.0, posinf=7.0))
    # without +inf nothing of this is left
    b[up] = 0.0
    r = reno.head_code_length(h.cuda(), w.cuda(), b.cuda(), s.cuda(), grad=grad)
    assert bool(r.lse.isfinite().all())
    # NaN beside +inf
    b[up], b[1] = math.inf, math.nan
    r = reno.head_code_length(h.cuda(), w.cuda(), b.cuda(), s.cuda())
    assert torch.equal(r.lse.isnan().cpu(), taken) and torch.equal(r.bits.isnan().cpu(), taken)
