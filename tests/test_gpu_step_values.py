"""The step after a gradient where single values tell: the moments' decay, squares past fp32, gradients and factors next
to the ends of the range; and lists of many tensors of a kind, tensors past 2^31 elements."""
import math

import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def half_step(x):
    """Half of the distance from |x| to the next fp32 value, for x in 64 bits."""
    a = x.abs().float()
    return (torch.nextafter(a, torch.full_like(a, math.inf)) - a).double() / 2


def state(n):
    return [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")], torch.zeros(2, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.95, 0.99), (0.3, 0.99999), (0.999, 0.999999), (0.0, 0.5)])
def test_moments_decay_by_beta(betas):
    """Without a gradient a moment is beta times what it was, rounded once.  The part of beta below fp32 is carried in
    fp32 (2^-24 of 2^-25), and so is its product with the moment."""
    g = torch.Generator().manual_seed(1)
    n = 5003
    m, v = torch.randn(n, generator=g).cuda(), torch.rand(n, generator=g).cuda() + 2.0 ** -10
    steps = torch.zeros(2, dtype=torch.int32, device="cuda")
    old = m.double(), v.double()
    say("decay", betas)
    reno.adamw_step([torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")], [m], [v], steps, betas=betas)
    for got, before, beta in zip((m, v), old, betas):
        want = beta * before
        assert bool(((got.double() - want).abs() <= half_step(want) + 2.0 ** -47 * before.abs()).all()), beta


def test_second_moment_of_many_steps():
    """The mean of exp_avg_sq over many elements after many steps.  Roundings of single elements have no sign (their mean
    over 4096 is below 2^-25 of it); what remains is the rounding of 1 - beta2, 2^-24."""
    n, beta2 = 4096, 0.999
    g = torch.Generator(device="cuda").manual_seed(2)
    w = [torch.zeros(n, device="cuda")]
    m, v, steps = state(n)
    v[0].fill_(1.0)
    want = v[0].double()
    for i in range(2000):
        x = torch.randn(n, generator=g, device="cuda")
        reno.adamw_step(w, [x], m, v, steps, lr=0.0, betas=(0.9, beta2))
        want = beta2 * want + (1 - beta2) * x.double().square()
    assert abs(float((v[0].double() / want - 1).mean())) <= 2.0 ** -22


@pytest.mark.parametrize("beta2,big", [(0.0, 1e20), (0.999, 1e21), (0.5, 1e21), (0.999, torch.finfo(F32).max),
                                       (0.0, torch.finfo(F32).max)])
def test_a_square_past_fp32_stops_its_element(beta2, big):
    """(1 - beta2) g^2 past fp32: exp_avg_sq is infinite and stays so, and the weight moves by its decay alone.  The
    elements beside it are as if it were not there."""
    n, lr, decay = 11, 0.25, 0.125
    w = [torch.full((n,), 2.0, device="cuda")]
    m, v, steps = state(n)
    other = [w[0].clone()]
    m1, v1, steps1 = state(n)
    want = 2.0
    for i in range(4):
        g = torch.full((n,), 0.5, device="cuda")
        reno.adamw_step(other, [g], m1, v1, steps1, lr=lr, betas=(0.9, beta2), weight_decay=decay)
        if i == 1:
            g[3], g[7] = big, -big
        reno.adamw_step(w, [g], m, v, steps, lr=lr, betas=(0.9, beta2), weight_decay=decay)
        if i == 0:
            want = float(w[0][3])
        else:
            want *= 1 - lr * decay
            for e in (3, 7):
                assert math.isinf(float(v[0][e])) and math.isfinite(float(m[0][e]))
                assert float(w[0][e]) == pytest.approx(want, rel=i * 2.0 ** -23)
        rest = [e for e in range(n) if e not in (3, 7)]
        assert torch.equal(w[0][rest], other[0][rest]) and torch.equal(v[0][rest], v1[0][rest])


@pytest.mark.parametrize("beta1", [0.9, 0.053])   # 0.053: the first moment over 1 - beta1 is rounded past fp32
def test_the_first_step_of_the_largest_gradient(beta1):
    w = [torch.ones(4, device="cuda")]
    m, v, steps = state(4)
    reno.adamw_step(w, [torch.full((4,), torch.finfo(F32).max, device="cuda")], m, v, steps, lr=0.5, betas=(beta1, 0.999),
                    weight_decay=0.25)
    assert bool(v[0].isinf().all()) and w[0].tolist() == [0.875] * 4


@pytest.mark.parametrize("scale", [1.0, 3.0, 0.7, 1e10, 2.0 ** 120, 1e60, 1e-10, 1e-30, 1e-60])
def test_clipping_rounds_once_anywhere(scale):
    """Gradients from the least fp32 value to the largest, factors in and out of the floats: the product is off by the
    rounding of the factor to 2^-24, and by half a step, that of subnormal values below 2^-126."""
    g = torch.Generator().manual_seed(4)
    x = torch.ldexp(1 + torch.rand(20000, generator=g, dtype=torch.float64), torch.randint(-149, 128, (20000,), generator=g))
    x = (x * torch.where(torch.rand(20000, generator=g) < 0.5, -1.0, 1.0)).float().cuda()
    for n, most in ((1.0, math.inf), (3.0, 1.0)):
        c = scale * min(1.0, most / n)
        say("clip, any size", scale, most)
        out = [torch.zeros_like(x)]
        reno.clip_grads([x], torch.tensor(n, device="cuda"), most, scale=scale, out=out)
        want = x.double() * c
        top = float(torch.finfo(F32).max)
        fits = want.abs() <= top * (1 - 2.0 ** -23)
        assert bool((out[0][want.abs() >= top * (1 + 2.0 ** -23)].isinf()).all())
        bound = (2.0 ** -24 * 1.01) * want.abs() + half_step(want.clamp(-top / 2, top / 2)).maximum(2.0 ** -25 * want.abs())
        bad = fits & ~((out[0].double() - want).abs() <= bound)
        assert not bool(bad.any()), (scale, most, x[bad][:3].tolist(), out[0][bad][:3].tolist(), want[bad][:3].tolist())


@pytest.mark.parametrize("kind", ["fp32", "bf16 copies"])
def test_adamw_of_many_tensors_of_a_kind(kind):
    """More tensors of one kind than a launch takes: each is updated once, and the step is counted once."""
    dt, count = (F32, 200) if kind == "fp32" else (BF16, 128)
    g = torch.Generator().manual_seed(6)
    w0 = [torch.randn(1 + 37 * (i % 9), generator=g).to(dt).cuda() for i in range(count)]
    grads = [torch.randn(t.shape, generator=g).to(dt).cuda() for t in w0]

    def run(lists):
        w = [t.clone() for t in w0]
        x = [[torch.zeros(t.shape, device="cuda") for t in w0] for _ in range(2)]
        c = [t.float() for t in w] if dt != F32 else None
        steps = [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in lists]
        for _ in range(3):
            for at, st in zip(lists, steps):
                reno.adamw_step(w[at], grads[at], x[0][at], x[1][at], st, master=c and c[at], lr=0.1)
        assert all(st.tolist() == [3, 0] for st in steps)
        return w, *x, c or []
    say("adamw, many", kind, count)
    one = run([slice(0, count)])
    each = run([slice(i, i + 1) for i in range(count)])
    assert all(torch.equal(a, b) for x, y in zip(one, each) for a, b in zip(x, y))


def test_adamw_past_31_bits():
    """Elements past 2^31, in the last of which and one before alone there is a gradient."""
    n = (1 << 31) + 4099
    w, g = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    steps = torch.zeros(2, dtype=torch.int32, device="cuda")
    g[-1], g[5] = 1.0, -1.0
    say("adamw, long", n)
    reno.adamw_step([w], [g], [m], [v], steps, lr=0.5, betas=(0.5, 0.5))
    # m / (1 - 0.5) = g, sqrt(v / (1 - 0.5)) = 1, eps is lost
    assert float(w[-1]) == -0.5 and float(w[5]) == 0.5 and steps.tolist() == [1, 0]
    assert float(m[-1]) == 0.5 and float(v[5]) == 0.5
    for t in (w, m, v):
        assert int(sum(torch.count_nonzero(x) for x in t.split(1 << 30))) == 2
