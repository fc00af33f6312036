"""Row weights at the ends of their range: what a row that is left out weighs
changes nothing of the others."""
import math

import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# 16 rows and fewer carry dz in two parts, the fp32 head of 200 symbols is a narrow one
SHAPES = [(90, 48, 300), (12, 48, 300), (90, 48, 200)]


def inputs(N, C, V, dt, seed):
    g = torch.Generator().manual_seed(seed + 7919 * N + 31 * C + V)
    h = torch.randn(N, C, generator=g).relu()
    w = torch.randn(C, V, generator=g) * math.sqrt(2.0 / C)
    b = torch.randn(V, generator=g) * 0.1
    s = torch.randint(0, V, (N,), generator=g).int()
    s[::3] = -1
    index = torch.randint(0, V, (N, 5), generator=g).int()
    index[::3] = -1
    logit = torch.randn(N, 5, generator=g)
    weight = 0.5 + torch.rand(N, generator=g)
    return [x.cuda() for x in (h.to(dt), w.to(dt), b.to(dt), s, index, logit, weight)]


def both(h, w, b, s, index, logit, weight):
    return [reno.head_code_length(h, w, b, s, row_weight=weight, grad=True),
            reno.head_distill(h, w, b, index, logit, temperature=1.5, row_weight=weight, grad=True)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V", SHAPES)
def test_weights_of_rows_left_out_change_nothing(N, C, V, dt):
    *x, weight = inputs(N, C, V, dt, 1)
    say("weights of rows left out", N, C, V, dt)
    weight[::3] = 0.0
    want = both(*x, weight)
    for low in (2.0 ** 24, 2.0 ** 60, 1e30, torch.finfo(torch.float32).max, math.inf, math.nan):
        weight[::3] = low
        weight[3] = -low
        for got, ref in zip(both(*x, weight), want):
            for name in ("bits", "lse", "dh", "dw", "db"):
                assert torch.equal(getattr(got, name), getattr(ref, name)), (low, name)
    assert all(bool(r.dw.any()) and bool(r.dh.any()) for r in want)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V", SHAPES)
def test_weights_of_rows_without_a_valid_target_stay_with_them(N, C, V, dt):
    """Their own gradient is NaN whatever they weigh; dh of the other rows is not theirs."""
    h, w, b, s, index, logit, weight = inputs(N, C, V, dt, 2)
    s[1], index[1, 2] = V, V + 5
    say("weights of rows outside", N, C, V, dt)
    want = both(h, w, b, s, index, logit, weight)
    weight[1] = 1e30
    for got, ref in zip(both(h, w, b, s, index, logit, weight), want):
        assert bool(got.dh[1].isnan().all()) and bool(got.dw.isnan().all())
        assert torch.equal(got.dh[2:], ref.dh[2:]) and bool(ref.dh[2:].any())
