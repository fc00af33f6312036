"""Rows' own temperatures past their range count as its end."""
import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say
from sample_ref import check, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [9, 40, 256, 300, 5000, 70001])
def test_temperatures_of_rows_past_their_range(V):
    N = 24
    g = torch.Generator().manual_seed(V)
    u = torch.rand(N, generator=g).cuda()
    steps = -torch.randint(0, 8, (N, V), generator=g).double()
    T = torch.tensor([1e-40, 2.0 ** -149, 2.0 ** -126, 2.0 ** -127] * 3 + [3e38, 1e38, 2.0 ** 126, 2.0 ** 127] * 3)
    z = torch.where(T[:, None] < 1, steps * 2.0 ** -128, steps * 5e36).float().cuda()
    ends = T.clamp(2.0 ** -126, 2.0 ** 126).cuda()
    for kw in (dict(), dict(top_p=0.6), dict(top_k=7), dict(top_k=V // 2 + 1, top_p=0.9), dict(min_p=0.3),
               dict(top_k=5, min_p=0.5, top_p=0.99)):
        say("sample, far rows", V, kw)
        got = reno.sample_symbols(z, u, temperature=T.cuda(), **kw)
        assert check(got, draw(z, u, temperature=ends, **kw), V, (V, kw)) >= N - 1
        want = reno.sample_symbols(z, u, temperature=ends, **kw)
        assert torch.equal(got.symbol, want.symbol) and torch.equal(got.bits, want.bits)
