"""Code length of a linear head with its gradient, and distillation from a
teacher's top logits, against the definitions in 64 bits within bounds that
count the roundings (head_ref)."""
import math

import numpy as np
import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say
from head_ref import check, reference, targets_of, targets_of_top

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SHAPES = [(1, 1, 1), (1, 16, 2), (3, 5, 7), (2, 64, 16), (17, 33, 65), (64, 32, 256), (87, 16, 256), (130, 128, 257),
          (257, 70, 1000), (33, 300, 513), (1025, 128, 130), (70, 1000, 2051), (700, 31, 16)]


def head_of(N, C, V, dt, seed=0, bias=True):
    g = torch.Generator().manual_seed(seed + 7919 * N + 31 * C + V)
    h = torch.randn(N, C, generator=g).relu()
    w = torch.randn(C, V, generator=g) * math.sqrt(2.0 / C)
    b = torch.randn(V, generator=g) * 0.1 if bias else None
    s = torch.randint(-1, V, (N,), generator=g).int()
    h = h + 2.0 * (torch.rand(N, 1, generator=g) < 0.5) * w.t()[s.long().clamp(min=0)]
    wt = 0.5 + torch.rand(N, generator=g)
    return h.to(dt), w.to(dt), None if b is None else b.to(dt), s, wt


def dev(*ts):
    return [None if t is None else t.cuda() for t in ts]


def top_of(N, V, k, seed=0):
    g = torch.Generator().manual_seed(seed + 13 * N + V + k)
    index = torch.rand(N, V, generator=g).topk(k, 1)[1].int() if V >= k else torch.randint(0, V, (N, k), generator=g).int()
    kept = torch.randint(0, k + 1, (N,), generator=g)
    index = torch.where(torch.arange(k) < torch.where(kept < k // 4, kept, k)[:, None], index, -1).int()
    return index, torch.randn(N, k, generator=g) * 3


def compare(r, ref, names=("bits", "lse", "dh", "dw", "db")):
    for x in names:
        check(x, getattr(r, x), *ref[x])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V", SHAPES)
def test_code_length(N, C, V, dt):
    say("head code length", N, C, V, dt)
    h, w, b, s, g = head_of(N, C, V, dt)
    ref = reference(h, w, b, *targets_of(s, V), g)
    r = reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True)
    compare(r, ref)
    f = reno.head_code_length(*dev(h, w, b, s))
    compare(f, ref, ("bits", "lse"))
    assert f.dh is None and f.dw is None and f.db is None


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V", [(1, 300, 1000), (2, 129, 300), (4, 200, 40000), (3, 4096, 33000), (1, 16384, 300),
                                   (2, 9000, 70), (5, 200, 400)])
def test_few_rows(N, C, V, dt):
    say("few rows", N, C, V, dt)
    h, w, b, s, _ = head_of(N, C, V, dt, seed=11)
    s[0] = V - 1
    if N > 2:
        s[1], h[1] = -1, math.nan
    ref = reference(h, w, b, *targets_of(s, V))
    compare(reno.head_code_length(*dev(h, w, b, s)), ref, ("bits", "lse"))
    # rows of w that do not start on 16 bytes
    wide = torch.full((C, V + 3), math.nan, dtype=dt, device="cuda")
    wide[:, 1:V + 1] = w.cuda()
    compare(reno.head_code_length(h.cuda(), wide[:, 1:V + 1], b.cuda(), s.cuda()), ref, ("bits", "lse"))
    index, logit = top_of(N, V, 70)
    compare(reno.head_distill(*dev(h.nan_to_num(0.0), w, b, index, logit), temperature=2.0),
            reference(h.nan_to_num(0.0), w, b, *targets_of_top(index, logit, 2.0, V), None, 2.0), ("bits", "lse"))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,C,V,k", [(600, 520, 20000, 1), (600, 520, 20001, 9), (4000, 4096, 300, 1), (130, 700, 9000, 33),
                                     (900, 96, 8008, 1)])
def test_large_tiles(N, C, V, k, dt):
    """Sizes that take the 256 x 256 tiles of each product, weights in place and packed, splits and none."""
    say("large tiles", N, C, V, k, dt)
    h, w, b, s, g = dev(*head_of(N, C, V, dt, seed=12))
    if k == 1:
        ref = reference(h, w, b, *targets_of(s, V), g)
        r = reno.head_code_length(h, w, b, s, row_weight=g, grad=True)
    else:
        index, logit = dev(*top_of(N, V, k))
        ref = reference(h, w, b, *targets_of_top(index, logit, 1.5, V), g, 1.5)
        r = reno.head_distill(h, w, b, index, logit, temperature=1.5, row_weight=g, grad=True)
    compare(r, ref)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("k,T", [(1, 1.0), (5, 2.0), (16, 1.0), (64, 0.5), (65, 1.0), (128, 4.0)])
@pytest.mark.parametrize("N,C,V", [(1, 3, 2), (87, 16, 256), (70, 130, 1001), (300, 40, 130)])
def test_distill(N, C, V, k, T, dt):
    say("head distill", N, C, V, dt, "k", k, "T", T)
    h, w, b, _, g = head_of(N, C, V, dt, seed=1)
    index, logit = top_of(N, V, k)
    ref = reference(h, w, b, *targets_of_top(index, logit, T, V), g, T)
    r = reno.head_distill(*dev(h, w, b, index, logit), temperature=T, row_weight=g.cuda(), grad=True)
    compare(r, ref)
    f = reno.head_distill(*dev(h, w, b, index, logit), temperature=T)
    compare(f, ref, ("bits", "lse"))


@pytest.mark.parametrize("dt", TYPES)
def test_rows_left_out_reach_nothing(dt):
    N, C, V = 90, 48, 300
    h, w, b, s, g = head_of(N, C, V, dt, seed=2)
    s[::3] = -1
    s[1] = -2 ** 31
    ref = reference(h, w, b, *targets_of(s, V), g)
    bad = h.clone()
    bad[::3] = math.nan
    bad[3] = math.inf
    bad[1] = torch.finfo(dt).min
    g2 = g.clone()
    g2[::3] = math.nan
    say("rows left out", dt)
    r = reno.head_code_length(*dev(bad, w, b, s), row_weight=g2.cuda(), grad=True)
    compare(r, ref)
    # all rows left out
    s[:] = -1
    r = reno.head_code_length(*dev(bad, w, b, s), row_weight=g2.cuda(), grad=True)
    for x in r:
        assert not bool(x.any())


@pytest.mark.parametrize("dt", TYPES)
def test_symbols_outside_the_alphabet_are_loud(dt):
    N, C, V = 40, 20, 100
    h, w, b, s, g = head_of(N, C, V, dt, seed=3)
    s[7], s[20] = V, 2 ** 31 - 1
    say("symbols outside", dt)
    r = reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True)
    nan = r.bits.isnan().cpu()
    assert nan[7] and nan[20] and int(nan.sum()) == 2
    assert bool(r.dh[7].isnan().all()) and bool(r.dw.isnan().all()) and bool(r.db.isnan().all())
    assert not bool(r.dh[8].isnan().any())
    index, logit = top_of(N, V, 5)
    index[3, 2] = V
    logit[4, 0], index[4, 0] = math.nan, 1
    logit[5, 0], index[5, 0] = math.inf, 1
    r = reno.head_distill(*dev(h, w, b, index, logit), grad=True)
    assert sorted(torch.nonzero(r.bits.isnan()).flatten().tolist()) == [3, 4, 5]


@pytest.mark.parametrize("dt", TYPES)
def test_masked_symbols(dt):
    """A bias of -inf (or the type's lowest value) takes a symbol out of the alphabet."""
    N, C, V = 50, 32, 270
    h, w, b, s, g = head_of(N, C, V, dt, seed=4)
    b[5::2] = -math.inf
    s = torch.where(s >= 0, s // 2 * 2, s).clamp(max=4 * (V // 5)).int()
    s[0], s[1] = 4, 7                       # a masked target costs infinitely many bits
    ref = reference(h, w, b, *targets_of(s, V), g)
    assert ref["bits"][0][1] == math.inf
    say("masked symbols", dt)
    r = reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True)
    compare(r, ref)
    b[5::2] = torch.finfo(dt).min / 4
    s[1] = 4
    ref = reference(h, w, b, *targets_of(s, V), g)
    compare(reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True), ref, ("lse", "dh", "dw", "db"))
    # a whole part of the alphabet, then all of it
    b[:] = 0
    b[:256] = -math.inf
    s[:] = 260
    ref = reference(h, w, b, *targets_of(s, V), g)
    compare(reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True), ref)
    # the rest far below zero
    for low in (-60.0, -200.0):
        b[256:] = low
        ref = reference(h, w, b, *targets_of(s, V), g)
        compare(reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True), ref)
    b[:] = -math.inf
    r = reno.head_code_length(*dev(h, w, b, s), grad=True)
    assert bool(r.bits.isnan().all()) and bool((r.lse == -math.inf).all())


@pytest.mark.parametrize("dt", TYPES)
def test_masked_parts_of_a_larger_alphabet(dt):
    """Parts of the alphabet without any symbol, beside logits far below zero."""
    N, C, V = 70, 40, 1100
    h, w, b, _, g = head_of(N, C, V, dt, seed=14)
    g_ = torch.Generator().manual_seed(2)
    for low in (0.0, -200.0, 90.0):
        b[:] = low
        b[64:640] = -math.inf
        b[1000:] = -math.inf
        s = torch.where(torch.rand(N, generator=g_) < 0.5, torch.randint(0, 64, (N,), generator=g_),
                        torch.randint(640, 1000, (N,), generator=g_)).int()
        s[3] = -1
        ref = reference(h, w, b, *targets_of(s, V), g)
        say("masked parts", dt, low)
        compare(reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True), ref)


@pytest.mark.parametrize("dt", TYPES)
def test_strides_alignment_and_no_bias(dt):
    N, C, V = 70, 64, 256
    h, w, _, s, g = head_of(N, C, V, dt, seed=5)
    ref = reference(h, w, None, *targets_of(s, V), g)
    for off, gap in ((0, 8), (1, 3), (3, 64)):
        hb = torch.full((N * (C + gap) + off,), math.nan, dtype=dt, device="cuda")
        wb = torch.full((C * (V + gap) + off,), math.nan, dtype=dt, device="cuda")
        hv = hb[off:].view(N, C + gap)[:, :C]
        wv = wb[off:].view(C, V + gap)[:, :V]
        hv.copy_(h)
        wv.copy_(w)
        say("strides", dt, off, gap)
        r = reno.head_code_length(hv, wv, None, s.cuda(), row_weight=g.cuda(), grad=True)
        compare(r, ref)
    # columns that are not contiguous, and rows that are one row
    hv = h.cuda().t().contiguous().t()
    compare(reno.head_code_length(hv, w.cuda(), None, s.cuda(), row_weight=g.cuda(), grad=True), ref)
    one = h[:1].expand(N, C)
    ref = reference(one, w, None, *targets_of(s, V), g)
    compare(reno.head_code_length(h[:1].cuda().expand(N, C), w.cuda(), None, s.cuda(), row_weight=g.cuda(), grad=True), ref)


@pytest.mark.parametrize("which", [("dh",), ("dw",), ("db",), ("dh", "db"), ("dw", "db")])
def test_some_gradients(which):
    N, C, V = 200, 32, 256
    h, w, b, s, g = head_of(N, C, V, torch.float32, seed=6)
    all_ = reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True)
    say("some gradients", which)
    r = reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=which)
    for x in ("dh", "dw", "db"):
        if x in which:
            assert torch.equal(getattr(r, x), getattr(all_, x))
        else:
            assert getattr(r, x) is None


@pytest.mark.parametrize("dt", TYPES)
def test_weights_of_any_size(dt):
    """The gradients scale with the row weights, however small or far apart these are; zero weights give zeros."""
    N, C, V = 100, 24, 256
    h, w, b, s, _ = head_of(N, C, V, dt, seed=7)
    for lo, hi in ((-60, -60), (40, 40), (-20, 6)) if dt != torch.float16 else ((-6, -6), (2, 2), (-10, 2)):
        g = torch.exp2(torch.linspace(lo, hi, N))
        ref = reference(h, w, b, *targets_of(s, V), g)
        say("weights", dt, lo, hi)
        compare(reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True), ref)
    r = reno.head_code_length(*dev(h, w, b, s), row_weight=torch.zeros(N).cuda(), grad=True)
    assert not bool(r.dh.any()) and not bool(r.dw.any()) and not bool(r.db.any())


def test_duplicates_and_empty_entries():
    N, C, V, k = 60, 20, 90, 12
    h, w, b, _, g = head_of(N, C, V, torch.float32, seed=8)
    gen = torch.Generator().manual_seed(3)
    index = torch.randint(-1, 6, (N, k), generator=gen).int()      # the same few symbols again and again
    logit = torch.randn(N, k, generator=gen) * 2
    logit[::4, ::2] = -math.inf
    logit[5] = -math.inf
    index[6] = -1
    ref = reference(h, w, b, *targets_of_top(index, logit, 1.0, V), g)
    assert not bool(targets_of_top(index, logit, 1.0, V)[1][5])
    say("duplicates")
    compare(reno.head_distill(*dev(h, w, b, index, logit), row_weight=g.cuda(), grad=True), ref)


def test_gradient_against_differences():
    """Central differences of the 64-bit loss in random directions."""
    N, C, V = 30, 20, 60
    h, w, b, s, g = head_of(N, C, V, torch.float32, seed=9)
    index, logit = top_of(N, V, 6)
    gen = torch.Generator().manual_seed(11)
    for kind in ("code", "distill"):
        if kind == "code":
            r = reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True)
            q, taken, bad = targets_of(s, V)
        else:
            r = reno.head_distill(*dev(h, w, b, index, logit), temperature=2.0, row_weight=g.cuda(), grad=True)
            q, taken, bad = targets_of_top(index, logit, 2.0, V)
        T = 1.0 if kind == "code" else 2.0

        def loss(hh, ww, bb):
            logp = torch.log_softmax((hh @ ww + bb) / T, 1)
            return float((-(q * logp).sum(1) * taken * g.double()).sum() / math.log(2.0))
        args = [h.double(), w.double(), b.double()]
        for i, name in enumerate(("dh", "dw", "db")):
            d = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
            step = 1e-5
            up = list(args)
            up[i] = args[i] + step * d
            down = list(args)
            down[i] = args[i] - step * d
            want = (loss(*up) - loss(*down)) / (2 * step)
            got = float((getattr(r, name).double().cpu() * d).sum())
            # differences: third derivatives of order 1 leave step^2 of the terms' size; gradients: fp32
            size = float((getattr(r, name).double().cpu() * d).abs().sum())
            assert abs(got - want) <= 1e-6 * size + 1e-7, (kind, name, got, want)


def test_no_rows():
    w, b = torch.randn(8, 20).cuda(), torch.randn(20).cuda()
    r = reno.head_code_length(torch.empty(0, 8).cuda(), w, b, torch.empty(0, dtype=torch.int32).cuda(), grad=True)
    assert r.bits.shape == (0,) and r.dh.shape == (0, 8)
    assert not bool(r.dw.any()) and not bool(r.db.any())
    r = reno.head_distill(torch.empty(0, 8).cuda(), w, b, torch.empty(0, 3, dtype=torch.int32).cuda(),
                          torch.empty(0, 3).cuda(), grad=True)
    assert not bool(r.dw.any()) and not bool(r.db.any())


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_pieces_of_rows(dt):
    """More logits than one piece holds: rows of several pieces add up in dw and db."""
    V, C = 40000, 24
    N = (1 << 27 if dt == torch.float32 else 1 << 28) // V + 301
    g = torch.Generator(device="cuda").manual_seed(5)
    h = torch.randn(N, C, generator=g, device="cuda").relu().to(dt)
    w = (torch.randn(C, V, generator=g, device="cuda") * math.sqrt(2.0 / C)).to(dt)
    b = (torch.randn(V, generator=g, device="cuda") * 0.1).to(dt)
    s = torch.randint(-1, V, (N,), generator=g, device="cuda").int()
    wt = torch.rand(N, generator=g, device="cuda") + 0.5
    say("pieces", N, C, V, dt)
    r = reno.head_code_length(h, w, b, s, row_weight=wt, grad=True)
    torch.cuda.synchronize()
    dw, edw, db, edb = 0.0, 0.0, 0.0, 0.0
    for i in range(0, N, 1024):
        e = slice(i, min(N, i + 1024))
        ref = reference(h[e], w, b, *targets_of(s[e], V), wt[e])
        for x in ("bits", "lse", "dh"):
            check(x, getattr(r, x)[e], *ref[x])
        dw, edw = dw + ref["dw"][0], edw + ref["dw"][1]
        db, edb = db + ref["db"][0], edb + ref["db"][1]
    # the bound of a piece of 1024 rows counts their sums; those of all N rows come on top
    more = (N + 16) * 2 * 2.0 ** -24
    check("dw", r.dw, dw, edw + more * (h.double().abs().T @ torch.ones(N, 1, device="cuda", dtype=torch.float64)))
    check("db", r.db, db, edb + more * N * 1.5 / V)


def test_features_past_32_bits():
    """Rows whose offset in h and dh passes 2^31 elements."""
    N, C, V, dt = 140000, 16384, 16, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(9)
    h = torch.randn(N, C, generator=g, device="cuda", dtype=dt)
    w = (torch.randn(C, V, generator=g, device="cuda") * math.sqrt(2.0 / C)).to(dt)
    b = torch.zeros(V, device="cuda", dtype=dt)
    s = torch.randint(-1, V, (N,), generator=g, device="cuda").int()
    say("features past 32 bits", N, C, V)
    r = reno.head_code_length(h, w, b, s, grad=True)
    torch.cuda.synchronize()
    dw, edw, size = 0.0, 0.0, 0.0
    for i in range(0, N, 20000):
        e = slice(i, min(N, i + 20000))
        ref = reference(h[e], w, b, *targets_of(s[e], V))
        for x in ("bits", "lse", "dh"):
            check(x, getattr(r, x)[e], *ref[x])
        dw, edw = dw + ref["dw"][0], edw + ref["dw"][1]
        size = size + h[e].double().abs().sum(0)
    # the bound of a part counts the sums of its 20000 rows; those of all N, with |dz| at most 1 / ln 2, come on top
    check("dw", r.dw, dw, edw + (N + 16) * 2 * 2.0 ** -24 / math.log(2.0) * size[:, None])


@pytest.mark.parametrize("N", [1, 2, 16, 17])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_few_rows_round_once(N, dt):
    """Up to 16 rows dz has two parts: beside the bound in 32 bits only the result is rounded."""
    C, V = 200, 700
    h, w, b, s, g = head_of(N, C, V, dt, seed=15)
    s = s.clamp(min=0)
    say("few rows round once", N, dt)
    r = reno.head_code_length(*dev(h, w, b, s), row_weight=g.cuda(), grad=True)
    ref = reference(h, w, b, *targets_of(s, V), g)
    compare(r, ref)
    if N <= 16:
        exact = reference(h.double().float(), w.float(), b.float(), *targets_of(s, V), g)   # bounds without the type
        u = torch.finfo(dt).eps / 2
        for x in ("dh", "dw", "db"):
            value, bound = exact[x]
            # dz in two parts of the type: 2^-16 (bf16), 2^-22 (fp16) of itself through the products' absolute values,
            # which the bound of the type's own rounding, u |dz|, gives divided by u and multiplied by u^2
            part = ref[x][1] * u * 2
            low = 2.0 ** -25 if dt == torch.float16 else 0.0
            check(x, getattr(r, x), value, bound + part + u * value.abs() * 1.01 + low)


@pytest.mark.parametrize("dt", TYPES)
def test_capture_streams_and_repeats(dt):
    N, C, V = 500, 64, 777
    h, w, b, s, g = dev(*head_of(N, C, V, dt, seed=10))
    index, logit = dev(*top_of(N, V, 9))
    want = reno.head_code_length(h, w, b, s, row_weight=g, grad=True)
    want2 = reno.head_distill(h, w, b, index, logit, temperature=1.5, row_weight=g, grad=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    say("capture", dt)
    with torch.cuda.graph(graph):
        r = reno.head_code_length(h, w, b, s, row_weight=g, grad=True)
        r2 = reno.head_distill(h, w, b, index, logit, temperature=1.5, row_weight=g, grad=True)
    h0 = h.clone()
    for i in range(4):
        for x in (*r, *r2):
            x.zero_()
        h.copy_(h0 * 0 if i == 2 else h0)
        graph.replay()
        torch.cuda.synchronize()
        same = all(torch.equal(x, y) for x, y in zip((*r, *r2), (*want, *want2)))
        assert same == (i != 2), i
    # another stream, two workspaces at once
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    need = reno.head_workspace(N, C, V, dt, 9, True)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    torch.cuda.synchronize()
    a = reno.head_distill(h, w, b, index, logit, temperature=1.5, row_weight=g, grad=True, workspace=ws, stream=st)
    c = reno.head_code_length(h, w, b, s, row_weight=g, grad=True)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((*c, *a), (*want, *want2)))


def test_refusals():
    h, w, b, s, g = dev(*head_of(10, 8, 20, torch.float32))
    call = reno.head_code_length
    index, logit = dev(*top_of(10, 20, 4))
    for bad in (lambda: call(h.double(), w.double(), b.double(), s), lambda: call(h, w.half(), b, s),
                lambda: call(h, w[:4], b, s), lambda: call(h, w, b[:3], s), lambda: call(h, w, b, s.long()),
                lambda: call(h, w, b, s[:5]), lambda: call(h, w, b, s.cpu()), lambda: call(h.cpu(), w, b, s),
                lambda: call(h, w, b, s, grad=("dx",)), lambda: call(h, w, b, s, row_weight=g[:3]),
                lambda: reno.head_distill(h, w, b, index, logit[:, :2]), lambda: reno.top_logits(h.long(), 2),
                lambda: reno.head_distill(h, w, b, index[:3], logit[:3])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call(h, w, b, s, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
                lambda: call(h, w, b, s, workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda")[8:]),
                lambda: reno.head_distill(h, w, b, index, logit, temperature=0.0),
                lambda: reno.head_distill(h, w, b, index, logit, temperature=math.nan),
                lambda: reno.top_logits(h, 0), lambda: reno.top_logits(h, 129)):
        with pytest.raises(reno.RenoError) as e:
            bad()
        assert e.value.status == reno.RENO_E_INVALID and str(e.value)
