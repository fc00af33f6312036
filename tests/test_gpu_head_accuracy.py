"""How exact the head's products are: relative 2-norms of the errors against 64
bits, at sizes where the sums are so short that a product's term, or the last
part of a sum, would be missed.

The element bounds of head_ref grow with the number of terms and leave room for
more than that.  Here a sum of S additions counts (2 S / 3 + 8) 2 eps, eps = 2^-24:
the matrix units may cut off (2 eps of a sum each), the sums before the last are
two thirds of it on average, 8 for the rest (splitting, exponentials, scaling).
fp32 operands are three bf16 parts each, cut off, and of the nine products the
three below 2^-21 of the whole are left out: 2^-24.6 of it on average.  The
smallest that is kept is x2 y0: 2^-17 of it at the mean (x2 lies evenly in 0 ..
2^-15 of x0, against mantissas from 1 to 2), 1e-5, so a term that is lost shows."""
import math

import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say
from head_ref import reference, targets_of, targets_of_top

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 2.0 ** -24


def sums(S):
    return (2 * S / 3 + 8) * 2 * EPS


def norm(got, want):
    return float((got.double() - want).norm() / want.norm())


def inputs(N, C, V, dt, seed, size=1.0):
    g = torch.Generator().manual_seed(seed + 7919 * N + 31 * C + V)
    h = torch.randn(N, C, generator=g)
    w = torch.randn(C, V, generator=g) * (size / math.sqrt(C))
    s = torch.randint(0, V, (N,), generator=g).int()
    wt = 0.5 + torch.rand(N, generator=g)
    return h.to(dt).cuda(), w.to(dt).cuda(), s.cuda(), wt.cuda()


# bits to 2 sqrt(2) of the logits' error (lse and the target's t), where both are of one size
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V", [(40, 64, 257), (200, 64, 300), (130, 32, 513), (300, 64, 200), (500, 128, 256),
                                   (3, 64, 300), (1, 64, 40000)])
def test_logits(N, C, V, dt):
    h, w, s, _ = inputs(N, C, V, dt, 1, 8.0)
    say("accuracy of the logits", N, C, V, dt)
    r = reno.head_code_length(h, w, None, s)
    ref = reference(h, w, None, *targets_of(s, V))
    z = h.double() @ w.double() / math.log(2.0)
    terms = 6 if dt == torch.float32 else 1
    few = N <= 4 and (dt != torch.float32 or V > 256)       # by vector instructions: one product, C / 4 in a chain at most
    chain = C / 4 + 16 if few else terms * C / 32
    # an error of e in a row's t moves lse and t by e; 4 eps |t| of the scaling, 4 eps of lse; over the bits' own norm
    t_norm = float((z.gather(1, s[:, None].long()).norm() ** 2 + z.amax(1).norm() ** 2) ** 0.5)
    most = (sums(chain) + 4 * EPS) * t_norm / float(ref["bits"][0].norm()) + 4 * EPS
    assert most < 6e-6 or few
    off = norm(r.bits, ref["bits"][0])
    assert off <= most, (off, most)
    off = norm(r.lse, ref["lse"][0])
    assert off <= (sums(chain) + 8 * EPS) * 1.5, off


def gradients(r, ref, dt, S):
    for x in ("dh", "dw", "db"):
        most = sums(S[x])
        if dt != torch.float32:
            # dz and the result rounded, each uniform in half a step of a value anywhere in its binade:
            # u sqrt(1/3) * 0.72, a quarter more for the spread of so few values
            most += torch.finfo(dt).eps / 2 * 0.415 * 1.4142 * 1.25
        off = norm(getattr(r, x), ref[x][0])
        assert off <= most, (x, off, most)


# dz is p - q, its norm that of q: an error of the logits reaches it only through p, 1 / V of it
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V", [(40, 64, 257), (128, 64, 300), (130, 300, 320), (64, 65, 321), (129, 128, 256),
                                   (129, 64, 250), (129, 32, 256)])
def test_gradients(N, C, V, dt):
    h, w, s, wt = inputs(N, C, V, dt, 2)
    say("accuracy of gradients", N, C, V, dt)
    r = reno.head_code_length(h, w, None, s, row_weight=wt, grad=True)
    ref = reference(h, w, None, *targets_of(s, V), wt)
    terms = 6 if dt == torch.float32 else 1
    gradients(r, ref, dt, {"dh": terms * (V + 63) // 64 * 2, "dw": terms * (N + 63) // 64 * 2, "db": N / 4 + 16})
    k = 3
    index = torch.stack([s, (s + 1) % V, (s + 7) % V], 1).int()
    logit = torch.randn(N, k, generator=torch.Generator().manual_seed(N)).cuda()
    r = reno.head_distill(h, w, None, index, logit, temperature=2.0, row_weight=wt, grad=True)
    ref = reference(h, w, None, *targets_of_top(index, logit, 2.0, V), wt, 2.0)
    gradients(r, ref, dt, {"dh": terms * (V + 63) // 64 * 2, "dw": terms * (N + 63) // 64 * 2, "db": N / 4 + 16})


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V", [(129, 65, 321), (257, 129, 1025), (200, 33, 66), (129, 33, 129), (641, 97, 193)])
def test_the_last_part_of_every_sum(N, C, V, dt):
    """Targets in the last symbols, channels and rows that are more than whole steps of 32 and 64: they carry the
    result, so that what drops them is off by all of it."""
    h, w, s, wt = inputs(N, C, V, dt, 3)
    h[:, :C // 32 * 32] *= 2.0 ** -8          # the last channels carry the logits
    w[:, :] = w * 4
    wt[:N // 32 * 32] = 2.0 ** -6             # the last rows the gradients of w
    s[:] = V // 32 * 32 + torch.arange(N, device="cuda").int() % (V % 32)
    say("the last part of sums", N, C, V, dt)
    r = reno.head_code_length(h, w, None, s, row_weight=wt, grad=True)
    ref = reference(h, w, None, *targets_of(s, V), wt)
    assert norm(r.bits, ref["bits"][0]) <= 1e-5 and norm(r.lse, ref["lse"][0]) <= 1e-5
    # without the last channels, symbols or rows nothing like this is left
    cut = h.clone()
    cut[:, C // 32 * 32:] = 0
    assert norm(reference(cut, w, None, *targets_of(s, V))["lse"][0], ref["lse"][0]) > 1e-2
    most = 1e-5 if dt == torch.float32 else 2 * torch.finfo(dt).eps
    for x in ("dh", "dw", "db"):
        off = norm(getattr(r, x), ref[x][0])
        assert off <= most, (x, off)


@pytest.mark.parametrize("C,V,k", [(33, 256, 0), (64, 256, 0), (128, 256, 0), (16, 16, 0), (128, 16, 0), (64, 64, 0),
                                   (32, 256, 20), (64, 256, 20), (128, 256, 20), (128, 200, 5), (20, 16, 17), (100, 60, 33)])
def test_many_rows_of_narrow_heads(C, V, k):
    """The narrow kernel's blocks take rows again and again: 16 rows a wave, 8 (up to 32 channels 4) waves a block and
    256 (512) blocks a turn; the last turn is ragged."""
    N = 2 * 32768 + 777
    h, w, s, wt = inputs(N, C, V, torch.float32, 4)
    s[::17] = -1
    h[::17] = math.nan
    b = torch.randn(V, generator=torch.Generator().manual_seed(V)).cuda() * 0.3
    say("many rows of narrow heads", C, V, k)
    if k:
        g = torch.Generator().manual_seed(k)
        index = torch.rand(N, V, generator=g).topk(min(k, V), 1)[1].int()
        index = torch.cat([index, torch.full((N, k - index.shape[1]), -1, dtype=torch.int32)], 1).cuda()
        index[::17] = -1
        logit = torch.randn(N, k, generator=g).cuda()
        r = reno.head_distill(h, w, b, index, logit, temperature=1.5, row_weight=wt, grad=True)
        f = reno.head_distill(h, w, b, index, logit, temperature=1.5)
        ref = reference(h, w, b, *targets_of_top(index, logit, 1.5, V), wt, 1.5)
    else:
        r = reno.head_code_length(h, w, b, s, row_weight=wt, grad=True)
        f = reno.head_code_length(h, w, b, s)
        ref = reference(h, w, b, *targets_of(s, V), wt)
    for x in ("bits", "lse", "dh", "dw", "db"):
        value, bound = ref[x]
        got = getattr(r, x).double()
        assert bool(((got - value).abs() <= bound).all()), x
        assert x[0] == "d" or bool(((getattr(f, x).double() - value).abs() <= bound).all()), x
    # dw: a block's rows (3 turns of 32, or 2 of 64 rows) in steps of 32, six products; 512 blocks in 16 shares
    assert norm(r.dh, ref["dh"][0]) <= sums(6 * 256 / 32) + 4 * EPS
    assert norm(r.dw, ref["dw"][0]) <= sums(6 * 3 * 4 + 48)
    assert norm(r.db, ref["db"][0]) <= sums(3 * 3 * 4 + 48)
