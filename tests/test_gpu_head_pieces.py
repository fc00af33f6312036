"""Calls whose rows are taken in several pieces: the pieces join in dw and db,
and targets, weights and results stay with their rows."""
import math

import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say
from head_ref import check, reference, targets_of, targets_of_top

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 2.0 ** -24


def inputs(N, C, V, dt, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(C, V, generator=g, device="cuda") * math.sqrt(2.0 / C)
    s = torch.randint(-1, V, (N,), generator=g, device="cuda").int()
    h = torch.empty(N, C, dtype=dt, device="cuda")
    for i in range(0, N, 1 << 17):
        e = slice(i, min(N, i + (1 << 17)))
        h[e] = torch.randn(e.stop - i, C, generator=g, device="cuda").relu().to(dt)
    b = (torch.randn(V, generator=g, device="cuda") * 0.1).to(dt)
    wt = torch.rand(N, generator=g, device="cuda") + 0.5
    index = torch.randint(-1, V, (N, max(k, 1)), generator=g, device="cuda").int()
    logit = torch.randn(N, max(k, 1), generator=g, device="cuda") * 2
    return h, w.to(dt), b, s, wt, index, logit


def by_slices(h, w, b, targets, wt, T, r, size, grad):
    """Checks every row of r; returns dw and db of all rows with their bounds."""
    N = h.shape[0]
    sums = {x: [0.0, 0.0] for x in ("dw", "db")}
    reach = [0.0, 0.0]
    for i in range(0, N, size):
        e = slice(i, min(N, i + size))
        q, taken, bad = targets(e)
        ref = reference(h[e], w, b, q, taken, bad, wt[e], T)
        for x in ("bits", "lse", "dh") if grad else ("bits", "lse"):
            check(x, getattr(r, x)[e], *ref[x])
        for x in sums:
            sums[x][0] = sums[x][0] + ref[x][0]
            sums[x][1] = sums[x][1] + ref[x][1]
        z = (torch.where(taken[:, None], h[e].double(), 0.0) @ w.double() + b.double()) / T
        dz = ((torch.softmax(z, 1) - q) * (taken * wt[e] / (T * math.log(2.0)))[:, None]).abs()
        reach[0] = reach[0] + h[e].double().abs().T @ dz
        reach[1] = reach[1] + dz.sum(0)
    # a slice's bound counts the sums of its rows; those of all N come on top: every one adds at most 2 eps of the sum
    # of the absolute values, of chains of at most N / 32 steps (k is taken 32 at a time) of up to six products
    chain = (6 * N / 32 + 600) * 2 * EPS
    return {x: (sums[x][0], sums[x][1] + chain * reach[j]) for j, x in enumerate(("dw", "db"))}


def close(x, got, want, rows, splits=1):
    """The 2-norm of the error, relative to that of the value: within what the roundings can add up to.

    fp32 sums: dw takes `rows` rows in steps of 32, six products each, and joins the splits one by one; db 64 rows in
    a wave, then every fourth wave of the others.  A sum is off by 2 eps of itself at most (the matrix units may cut
    off), and the sums before the last are two thirds of it on average where they grow evenly or slower.
    16-bit gradients: two more roundings, of dz and of the result, uniform in half a step u of a value anywhere in its
    binade: u sqrt(1/3) * 0.72 (the mean of 1 / mantissa), a quarter more for their spread."""
    chain = 6 * rows / 32 + splits if x == "dw" else 64 + rows * splits / 256
    most = (2 / 3 * chain + 8) * 2 * EPS
    if got.dtype != torch.float32:
        most += torch.finfo(got.dtype).eps / 2 * 0.415 * 1.4142 * 1.25
    off = float((got.double() - want).norm() / want.norm())
    assert off <= most, (x, off, most)


def in_range(got, want):
    """A gradient past its type is infinite (within 1 % of the type's largest: either); elsewhere both as they are."""
    most = torch.finfo(got.dtype).max
    over = want.abs() > 1.01 * most
    assert bool((got[over].double() == torch.sign(want[over]) * math.inf).all())
    over = want.abs() > 0.99 * most
    return torch.where(over, 0.0, got.double()).to(got.dtype), torch.where(over, 0.0, want)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_distill_over_pieces_of_logits(dt):
    """2^28 (2^27) logits and more: two pieces, several entries a row."""
    V, C, k, T = 40000, 24, 9, 1.5
    N = (1 << 27 if dt == torch.float32 else 1 << 28) // V + 301
    h, w, b, _, wt, index, logit = inputs(N, C, V, dt, k, 1)
    say("distill over pieces", N, C, V, dt)
    r = reno.head_distill(h, w, b, index, logit, temperature=T, row_weight=wt, grad=True)
    torch.cuda.synchronize()
    ref = by_slices(h, w, b, lambda e: targets_of_top(index[e], logit[e], T, V), wt, T, r, 1024, True)
    for x in ("dw", "db"):
        check(x, getattr(r, x), *ref[x])
        close(x, getattr(r, x), ref[x][0], N)


@pytest.mark.parametrize("dt", TYPES)
def test_splits_over_pieces(dt):
    """Few symbols: dw takes one tile, its rows are split, and there are two pieces of them."""
    V, C = 16, 130
    N = (1 << 27 if dt == torch.float32 else 1 << 28) // 64 + 301
    h, w, b, s, wt, _, _ = inputs(N, C, V, dt, 0, 2)
    say("splits over pieces", N, C, V, dt)
    r = reno.head_code_length(h, w, b, s, row_weight=wt, grad=True)
    torch.cuda.synchronize()
    ref = by_slices(h, w, b, lambda e: targets_of(s[e], V), wt, 1.0, r, 1 << 19, True)
    for x in ("dw", "db"):
        got, want = in_range(getattr(r, x), ref[x][0])
        check(x, got, want, ref[x][1])
        close(x, got, want, N // 512, 512)
    only = reno.head_code_length(h, w, b, s, row_weight=wt)
    assert torch.equal(only.lse, r.lse) and torch.equal(only.bits, r.bits)


@pytest.mark.parametrize("grad", [False, True])
def test_pieces_of_wide_rows(grad):
    """Few symbols and many channels: the pieces are bounded by the copy of h."""
    N, C, V, k, T = 22100, 16384, 20, 3, 2.0
    dt = torch.float32
    h, w, b, _, wt, index, logit = inputs(N, C, V, dt, k, 3)
    say("pieces of wide rows", N, C, V, grad)
    r = reno.head_distill(h, w, b, index, logit, temperature=T, row_weight=wt, grad=grad)
    torch.cuda.synchronize()
    ref = by_slices(h, w, b, lambda e: targets_of_top(index[e], logit[e], T, V), wt, T, r, 4096, grad)
    for x in ("dw", "db") if grad else ():
        check(x, getattr(r, x), *ref[x])
        close(x, getattr(r, x), ref[x][0], N)
