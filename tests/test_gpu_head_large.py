"""The largest sizes: operands whose elements pass 2^31, rows that one launch
does not take."""
import math

import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say
from head_ref import check, reference, targets_of, targets_of_top

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


# in place; copied (rows of w off 16 bytes); fp32; up to 4 rows without gradients by the vector kernel
@pytest.mark.parametrize("N,V,dt", [(20, 1 << 20, torch.bfloat16), (5, (1 << 20) - 3, torch.float16),
                                    (18, (1 << 20) - 1, torch.float32)])
def test_weights_past_32_bits(N, V, dt):
    C = (1 << 31) // V + 2
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(C, V, dtype=dt, device="cuda")
    for c in range(0, C, 256):
        w[c:c + 256] = (torch.randn(min(256, C - c), V, generator=g, device="cuda") * math.sqrt(2.0 / C)).to(dt)
    w[C - 2:] *= 16                                # the channels past 2^31 carry the logits
    h = torch.randn(N, C, generator=g, device="cuda").to(dt)
    s = torch.randint(0, V, (N,), generator=g, device="cuda").int()
    s[0], s[N - 1] = V - 1, -1
    say("weights past 32 bits", N, C, V, dt)
    r = reno.head_code_length(h, w, None, s, grad=True)
    few = reno.head_code_length(h[:2], w, None, s[:2])
    torch.cuda.synchronize()
    u = torch.finfo(dt).eps / 2
    z = torch.empty(N, V, dtype=torch.float64, device="cuda")
    for v in range(0, V, 1 << 16):
        z[:, v:v + (1 << 16)] = h.double() @ w[:, v:v + (1 << 16)].double()
    z[N - 1] = 0
    lse = torch.logsumexp(z, 1)
    taken = (s >= 0)
    bits = torch.where(taken, (lse - z.gather(1, s.long().clamp(min=0)[:, None])[:, 0]) / math.log(2.0), 0.0)
    # logits: a chain of C / 32 steps (fp32: of six products), (2 S / 3 + 8) 2 eps of the largest; sums of 2^20
    # exponentials in chains of 16 + V / 1024
    S = (6 if dt == torch.float32 else 1) * C / 32
    near = (2 * S / 3 + 8) * 2 * EPS * float(z.abs().amax()) + (16 + V / 1024) * 2 * EPS
    assert near < 2e-3
    assert bool(((r.bits.double() - bits).abs() <= 4 * near).all())
    assert bool(((r.lse.double() - torch.where(taken, lse, 0.0)).abs() <= 4 * near).all())
    assert bool(((few.bits.double() - bits[:2]).abs() <= 4 * near).all())
    dz = torch.exp(z - lse[:, None])
    dz[torch.arange(N, device="cuda"), s.long().clamp(min=0)] -= 1.0
    dz *= taken[:, None] / math.log(2.0)
    # gradients by norm and by the channels at the end: two roundings to the type (fp32: its sums), logits' error in p
    most = 4 * u + 8 * near
    dh = torch.zeros(N, C, dtype=torch.float64, device="cuda")
    for v in range(0, V, 1 << 16):
        dh += dz[:, v:v + (1 << 16)] @ w[:, v:v + (1 << 16)].double().T
    assert float((r.dh.double() - dh).norm() / dh.norm()) <= most
    assert float((r.dh[:, C - 2:].double() - dh[:, C - 2:]).norm() / dh[:, C - 2:].norm()) <= most
    low = 2.0 ** -25 if dt == torch.float16 else 0.0
    for c in (0, C // 2, C - 2):
        want = h[:, c:c + 2].double().T @ dz
        off = (r.dw[c:c + 2].double() - want).clamp(min=low).sub(low) if low else r.dw[c:c + 2].double() - want
        assert float(off.norm() / want.norm()) <= most, c
    want = dz.sum(0)
    assert float((r.db.double() - want).norm() / want.norm()) <= most


def test_narrow_rows_past_32_bits():
    """Elements of h and dh past 2^31 in the narrow kernel, and more rows than one launch of the targets takes."""
    N, C, V, k = (1 << 24) + 9, 128, 16, 2
    g = torch.Generator(device="cuda").manual_seed(2)
    h = torch.empty(N, C, device="cuda")
    for i in range(0, N, 1 << 21):
        h[i:i + (1 << 21)] = torch.randn(min(1 << 21, N - i), C, generator=g, device="cuda")
    w = torch.randn(C, V, generator=g, device="cuda") * math.sqrt(2.0 / C)
    b = torch.randn(V, generator=g, device="cuda") * 0.1
    index = torch.randint(-1, V, (N, k), generator=g, device="cuda", dtype=torch.int32)
    logit = torch.randn(N, k, generator=g, device="cuda")
    say("narrow rows past 32 bits", N, C, V)
    r = reno.head_distill(h, w, b, index, logit, temperature=2.0, grad=True)
    torch.cuda.synchronize()
    dw, db = 0.0, 0.0
    for i in range(0, N, 1 << 20):
        e = slice(i, min(N, i + (1 << 20)))
        ref = reference(h[e], w, b, *targets_of_top(index[e], logit[e], 2.0, V), None, 2.0)
        for x in ("bits", "lse", "dh"):
            value, bound = ref[x]
            assert bool(((getattr(r, x)[e].double() - value).abs() <= bound).all()), (x, i)
        dw, db = dw + ref["dw"][0], db + ref["db"][0]
    # sums of 256 blocks' (C > 32) rows of 32 in turn, six products: (2 S / 3 + 8) 2 eps
    S = 6 * N / 256 / 32 + 32
    assert float((r.dw.double() - dw).norm() / dw.norm()) <= (2 * S / 3 + 8) * 2 * EPS
    assert float((r.db.double() - db).norm() / db.norm()) <= (2 * S / 3 + 8) * 2 * EPS


@pytest.mark.parametrize("V,k,dt", [(3, 2, torch.float32), (16, 5, torch.bfloat16), (257, 3, torch.float16)])
def test_top_logits_of_more_rows_than_a_launch(V, k, dt):
    N = (1 << 21) + 33
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(N, V, generator=g, device="cuda").to(dt)
    say("top logits of many rows", N, V, k, dt)
    r = reno.top_logits(x, k)
    value, index = torch.sort(x.float(), dim=1, descending=True, stable=True)
    assert torch.equal(r.value, value[:, :k]) and torch.equal(r.index, index[:, :k].int())
    lse = torch.logsumexp(x.double(), 1)
    assert bool(((r.lse.double() - lse).abs() <= (4 + 2 * 90 + 64 + V / 64) * 2 * EPS + 4 * EPS * lse.abs()).all())


def test_long_rows_of_logits_are_their_own():
    """Values of rows whose offset passes 2^31 elements: each row has its own."""
    V = 1 << 20
    N = (1 << 31) // V + 3
    x = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    i = torch.arange(N, device="cuda")
    first, second = (i % 251 + 2).to(torch.bfloat16), ((i * 7) % 241 / 256).to(torch.bfloat16) + 1
    at = (i * 509) % (V // 2)
    x[i, at], x[i, V // 2 + at] = first, second
    say("top logits, rows past 32 bits", N, V)
    r = reno.top_logits(x, 3)
    assert torch.equal(r.value[:, 0], first.float()) and torch.equal(r.value[:, 1], second.float())
    assert torch.equal(r.index[:, 0].long(), at) and torch.equal(r.index[:, 1].long(), V // 2 + at)
    assert not bool(r.value[:, 2].any()) and torch.equal(r.index[:, 2].long(), (at == 0).long())
    lse = torch.log(torch.exp(first.double()) + torch.exp(second.double()) + (V - 2))
    assert bool(((r.lse.double() - lse).abs() <= (4 + 2 * 500 + 64 + V / 64) * 2 * EPS + 4 * EPS * lse).all())
