"""Row weights and temperatures at the ends of their ranges: what a row that is
left out weighs changes nothing of the others, and gradients whose weight over
the temperature lies far from 1 keep their bits."""
import math

import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say
from head_ref import check, reference, targets_of_top

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


@pytest.mark.parametrize("V", [300])
def test_large_weights_at_a_low_temperature(V):
    """g / T is past the largest float, dh = g / (T ln 2) sum (p - q) w is not."""
    N, C, T, G = 40, 48, 2.0 ** -100, 2.0 ** 40
    h, w, _, _, index, logit, weight = inputs(N, C, V, torch.float32, 3)
    h, w, logit, weight = h * 2.0 ** -10, w * 2.0 ** -90, logit * T, weight * G
    say("large weights, low temperature", V)
    r = reno.head_distill(h, w, None, index, logit, temperature=T, row_weight=weight, grad=("dh",))
    ref = reference(h, w, None, *targets_of_top(index, logit, T, V), weight, T)
    assert 2.0 ** 40 < float(ref["dh"][0].abs().max()) < 2.0 ** 60
    for x in ("bits", "dh"):
        check(x, getattr(r, x), *ref[x])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [300])
def test_gradients_of_zero_at_a_low_temperature(V, dt):
    """One symbol's worth of teacher and student: p - q is 0, and so is every gradient, however large g / T."""
    N, C, T = 20, 48, 2.0 ** -100
    h = torch.ones(N, C, dtype=dt, device="cuda")
    w = torch.zeros(C, V, dtype=dt, device="cuda")
    b = torch.full((V,), -math.inf, dtype=dt, device="cuda")
    b[7] = 0.0
    index = torch.full((N, 1), 7, dtype=torch.int32, device="cuda")
    weight = torch.full((N,), 2.0 ** 40, device="cuda")
    say("gradients of zero", V, dt)
    r = reno.head_distill(h, w, b, index, torch.zeros(N, 1, device="cuda"), temperature=T, row_weight=weight, grad=True)
    for x in (r.bits, r.dh, r.dw, r.db):
        assert not bool(x.any())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_large_weights_at_a_high_temperature(dt):
    """1 / (T ln 2) over fp16's 2^14 lies below the normal floats, the gradients do not."""
    N, C, V = 16, 48, 300
    T = float(torch.tensor(2.0 ** 135 / (math.log(2.0) * 530.5), dtype=torch.float32))   # half a step between two of them
    h, w, b, _, index, logit, weight = inputs(N, C, V, dt, 4)
    weight = weight * 2.0 ** 125
    say("large weights, high temperature", dt)
    r = reno.head_distill(h, w, b, index, logit, temperature=T, row_weight=weight, grad=True)
    q, taken, bad = targets_of_top(index, logit, T, V)
    exact = reference(h.float(), w.float(), b.float(), q, taken, bad, weight, T)
    # of the type's: the result's rounding, and dz in two parts (2^-16 of itself, fp16 2^-22) through |w| and |h|
    u = torch.finfo(dt).eps / 2
    dz = (weight.double() / (T * math.log(2.0)))[:, None] * (1.0 / V - q).abs() * 1.01 * taken[:, None]
    part = {"dh": dz @ w.double().abs().T, "dw": h.double().abs().T @ dz, "db": 0.0}
    for x in ("dh", "dw", "db"):
        value, bound = exact[x]
        check(x, getattr(r, x), value, bound + 2 * u * u * part[x] + u * value.abs() * 1.01 + 2.0 ** -25)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [300])
def test_weights_at_the_ends_of_fp32(V, dt):
    """The largest float and the smallest normal one as every row's weight, brought to size by the temperature."""
    N, C = 40, 48
    h, w, b, _, index, logit, weight = inputs(N, C, V, dt, 5)
    for e, T in ((126.9, 2.0 ** 125), (-125.0, 2.0 ** -120)):
        scale = 1.0 if T > 1 else 2.0 ** -60 if dt == torch.float32 else 0.0   # logits of 0 where T leaves no others
        weight = torch.full((N,), 2.0 ** e, device="cuda")
        a, c = (h * scale).to(dt), (w * scale if scale else w).to(dt)
        say("weights at the ends", V, dt, e)
        r = reno.head_distill(a, c, None, index, logit * min(T, 1.0), temperature=T, row_weight=weight, grad=True)
        ref = reference(a, c, None, *targets_of_top(index, logit * min(T, 1.0), T, V), weight, T)
        for x in ("bits", "dh", "dw", "db"):
            check(x, getattr(r, x), *ref[x])


@pytest.mark.parametrize("C", [24, 48, 128])
@pytest.mark.parametrize("e,T", [(126.9, 2.0 ** 125), (-125.0, 2.0 ** -120), (40.0, 2.0 ** -100), (-100.0, 2.0 ** -90)])
def test_narrow_heads_at_the_ends_of_fp32(C, e, T):
    N, V = 300, 200
    h, w, b, _, index, logit, _ = inputs(N, C, V, torch.float32, 6)
    weight = torch.full((N,), 2.0 ** e, device="cuda")
    scale = 1.0 if T > 1 else math.sqrt(T)       # logits of order 1 over T
    h, w, logit = h * scale, w * scale, logit * min(T, 1.0)
    say("narrow heads at the ends", C, e, T)
    r = reno.head_distill(h, w, None, index, logit, temperature=T, row_weight=weight, grad=True)
    ref = reference(h, w, None, *targets_of_top(index, logit, T, V), weight, T)
    big = torch.finfo(torch.float32).max
    for x in ("bits", "dh", "dw", "db"):
        value, bound = ref[x]
        over = value.abs() > big                 # past fp32: infinite
        assert bool((getattr(r, x)[over].abs() == math.inf).all()) and not (x == "dh" and bool(over.any()))
        check(x, torch.where(over, 0.0, getattr(r, x).double()), torch.where(over, 0.0, value), bound)


def test_narrow_gradients_of_zero_at_a_low_temperature():
    test_gradients_of_zero_at_a_low_temperature(200, torch.float32)
    test_large_weights_at_a_low_temperature(200)
    test_weights_at_the_ends_of_fp32(200, torch.float32)
