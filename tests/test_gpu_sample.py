"""Symbols drawn from logits against the definition in 64 bits: sizes, types, settings of all rows and of each, masks,
ties, infinities, strides, streams, graphs; then draws as the codec's decoder continues a frame with them."""
import math

import numpy as np
import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import cfg_dict, encode, make_ctx, say
from sample_ref import check, draw
from synth import CONFIGS, gen_weights

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 1), (7, 2), (5, 15), (33, 16), (19, 17), (9, 100), (37, 255), (130, 256), (7, 257), (5, 1000), (3, 2049),
         (4, 8191), (2, 20001), (2, 50021), (1, 131071)]
SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=1), dict(top_k=5), dict(top_p=0.9),
            dict(temperature=1.5, top_p=0.5), dict(min_p=0.05), dict(temperature=0.8, top_k=50, top_p=0.95),
            dict(top_k=20, top_p=0.3, min_p=0.02), dict(top_p=0.0), dict(top_p=0.999, min_p=1e-4), dict(min_p=1.0),
            dict(temperature=2.0, top_k=10 ** 9)]


def make(N, V, dt, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(N, V, generator=g) * spread).to(dt).cuda(), torch.rand(N, generator=g).cuda()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("N,V", SIZES)
def test_sizes_and_settings(N, V, dt):
    for i, kw in enumerate(SETTINGS):
        z, u = make(N, V, dt, 1000 * V + i)
        say("sample", N, V, dt, kw)
        got = reno.sample_symbols(z, u, **kw)
        assert check(got, draw(z, u, **kw), V, (N, V, dt, kw)) >= N - 1
        again = reno.sample_symbols(z, u, **kw)
        assert torch.equal(got.symbol, again.symbol) and torch.equal(got.bits, again.bits)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [16, 255, 256, 900, 5003, 40007])
def test_settings_of_each_row(V, dt):
    N = 24
    g = torch.Generator().manual_seed(V)
    z, u = make(N, V, dt, V + 1)
    T = torch.rand(N, generator=g) * 2
    T[::6] = 0.0
    k = torch.randint(-2, V + 3, (N,), generator=g).int()
    k[::2] = torch.randint(1, 9, (N // 2,), generator=g).int()
    p = torch.rand(N, generator=g)
    p[1::5] = 1.0
    p[2::7] = -0.5
    p[3::7] = 1.5
    least = torch.rand(N, generator=g) ** 4
    least[::3] = 0.0
    least[4] = 2.0
    allowed = torch.rand(N, V, generator=g) < torch.rand(N, 1, generator=g)
    allowed[7] = False
    kw = dict(temperature=T.cuda(), top_k=k.cuda(), top_p=p.cuda(), min_p=least.cuda())
    for a in (None, allowed[3].cuda(), allowed.cuda()):
        say("sample, each row", V, dt, None if a is None else tuple(a.shape))
        assert check(reno.sample_symbols(z, u, allowed=a, **kw), draw(z, u, allowed=a, **kw), V, (V, dt)) >= N - 1
    # what is no setting: symbol -1, NaN bits
    T[0], T[1], T[2], p[3], least[4] = -1.0, math.inf, math.nan, math.nan, math.nan
    kw = dict(temperature=T.cuda(), top_k=k.cuda(), top_p=p.cuda(), min_p=least.cuda())
    r = reno.sample_symbols(z, u, **kw)
    assert r.symbol[:5].tolist() == [-1] * 5 and bool(r.bits[:5].isnan().all())
    check(r, draw(z, u, **kw), V, (V, dt))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [16, 64, 256, 3000, 70001])
def test_ties_infinities_masks(V, dt):
    N = 20
    g = torch.Generator().manual_seed(V)
    x = torch.randint(-2, 3, (N, V), generator=g).to(dt)   # runs of equal logits, cut within
    allowed = torch.ones(N, V, dtype=torch.bool)
    x[1] = 0.0
    x[1, ::2] = -0.0                    # equal zeros of both signs
    x[2] = -math.inf                    # no symbol
    x[3] = -math.inf
    x[3, V // 2] = 1.0                  # one
    x[4, 5] = math.inf                  # no distribution
    x[5, 7] = math.nan
    x[6] = torch.finfo(dt).min          # equal lowest values: uniform
    x[7] = torch.finfo(dt).min
    x[7, 3] = 0.0
    x[7, V - 1] = 0.5
    x[8, 5] = math.inf
    x[8, 9] = math.nan
    x[8, 11] = -math.nan
    allowed[8, [5, 9, 11]] = False      # where they are masked they count for nothing
    x[9] = math.nan
    allowed[9] = False                  # nothing is left
    x[10] = torch.arange(V, 0, -1).to(dt)
    x[11] = torch.arange(V).to(dt)
    x[12] = torch.finfo(dt).max
    x[13, ::2] = torch.finfo(dt).max
    x[13, 1::2] = torch.finfo(dt).min
    allowed[14] = False
    allowed[14, V - 1] = True
    x[15] = 0.0
    x[15, V - 1] = 60.0 if dt != torch.float16 else 30.0
    u = torch.rand(N, generator=g)
    u[16], u[17], u[18], u[19] = -1.0, 1.0, math.nan, math.inf   # left out
    for seed, kw in enumerate(SETTINGS + [dict(top_p=0.5), dict(top_k=V // 2 + 1), dict(top_k=V // 3 + 1, top_p=0.6)]):
        for special in (False, True):
            uu = u.clone()
            if special:
                uu[:16] = torch.tensor([0.0, 1 - 2.0 ** -24] * 8)
            say("sample, ties", V, dt, kw, special)
            args = (x.cuda(), uu.cuda())
            r = reno.sample_symbols(*args, allowed=allowed.cuda(), **kw)
            check(r, draw(*args, allowed=allowed, **kw), V, (V, dt, kw, special))
            assert r.symbol[[2, 9]].tolist() == [-1, -1] and r.bits[[2, 9]].tolist() == [0.0, 0.0]
            assert r.symbol[[4, 5]].tolist() == [-1, -1] and bool(r.bits[[4, 5]].isnan().all())
            assert r.symbol[16:].tolist() == [-1] * 4 and r.bits[16:].tolist() == [0.0] * 4


def test_uniform_borders_are_exact():
    """Equal weights: u V and p V are whole where both are dyadic, and the sums that meet them are exact."""
    for V in (16, 256, 4096, 65536):
        N = 64
        z = torch.full((N, V), 1.25).cuda()
        u = (torch.arange(N) / N).cuda()
        r = reno.sample_symbols(z, u)
        assert r.symbol.cpu().tolist() == [i * V // N for i in range(N)]
        assert bool((r.bits == math.log2(V)).all())
        r = reno.sample_symbols(z, u, top_p=0.25)   # the first quarter by index
        assert r.symbol.cpu().tolist() == [i * (V // 4) // N for i in range(N)]
        r = reno.sample_symbols(z, u, top_k=3)
        assert r.symbol.cpu().tolist() == [int(i / N * 3) for i in range(N)]


def test_far_temperatures_and_small_weights():
    V = 300
    z, u = make(40, V, torch.float32, 5)
    for T in (2.0 ** -126, 1e-30, 1e-3, 1e4, 1e30, 2.0 ** 126):
        for kw in (dict(), dict(top_p=0.7), dict(top_k=9, top_p=0.4)):
            say("sample, temperature", T, kw)
            check(reno.sample_symbols(z, u, temperature=T, **kw), draw(z, u, temperature=T, **kw), V, (T, kw))
    # a u of 0 draws the first symbol that has any weight, however small
    z = torch.full((4, V), -math.inf)
    z[:, 40] = 0.0
    z[0, 7] = -300.0
    z[1, 7] = -600.0
    z[2, 7] = -5000.0       # exp of it is 0
    z[3, 7] = -math.inf
    r = reno.sample_symbols(z.cuda(), torch.zeros(4).cuda())
    assert r.symbol.tolist() == [7, 7, 40, 40]
    assert r.bits[0].item() == pytest.approx(300 / math.log(2), rel=2.0 ** -23)


@pytest.mark.parametrize("dt", TYPES)
def test_strides(dt):
    N, V = 20, 300
    for off, gap in ((0, 4), (1, 1), (3, 213)):
        buf = torch.full((N * (V + gap) + off,), 1e4, device="cuda").to(dt)
        z = buf[off:].view(N, V + gap)[:, :V]
        z.copy_(torch.randn(N, V, generator=torch.Generator().manual_seed(off)))
        mbuf = torch.ones(N * (V + gap) + off, dtype=torch.bool, device="cuda")
        allowed = mbuf[off:].view(N, V + gap)[:, :V]
        allowed.copy_(torch.rand(N, V, generator=torch.Generator().manual_seed(off + 1)) < 0.5)
        u = torch.rand(2 * N, generator=torch.Generator().manual_seed(off + 2)).cuda()[::2]
        say("sample, strided", off, gap, dt)
        assert check(reno.sample_symbols(z, u, top_p=0.9, allowed=allowed), draw(z, u, top_p=0.9, allowed=allowed), V) == N
        zt = z.t().contiguous().t()    # columns: copied
        assert torch.equal(reno.sample_symbols(zt, u, top_p=0.9).symbol, reno.sample_symbols(z, u, top_p=0.9).symbol)
    r = reno.sample_symbols(buf[:0].view(0, 9), torch.empty(0, device="cuda"))
    assert r.symbol.shape == (0,) and r.bits.shape == (0,)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", [257, 600, 1100, 2100, 4200, 9000, 33000, 66000])
def test_many_rows(V, dt):
    """More rows than CUs: other numbers of threads a row."""
    N = 260
    g = torch.Generator().manual_seed(V)
    z, u = make(N, V, dt, V + 7)
    z[:, 5] = -math.inf
    z[3] = 0.0                          # one value
    z[4, V // 2:] = 0.0                 # many logits of a value that is in no table
    z[5] = z[5] * 0.001                 # all of them small
    z[6] = z[6] * 40                    # far beyond
    z[7, 9] = 90.0 if dt != torch.float16 else 60.0
    z[8] = z[8].abs() * -1 - 3
    z[9, 1] = math.nan
    z[10, V - 1] = math.inf
    z[11] = -math.inf
    p = torch.rand(N, generator=g)
    p[:20] = 0.9
    k = torch.zeros(N, dtype=torch.int32)
    k[100:180] = torch.randint(1, V, (80,), generator=g).int()
    k[180:] = torch.randint(1, 300, (80,), generator=g).int()
    p[100:140] = 1.0
    least = torch.where(torch.rand(N, generator=g) < 0.2, 0.01, 0.0)
    for kw in (dict(top_p=0.9), dict(top_p=p.cuda(), top_k=k.cuda(), min_p=least.cuda()), dict()):
        say("sample, many rows", V, dt, sorted(kw))
        assert check(reno.sample_symbols(z, u, **kw), draw(z, u, **kw), V, (V, dt, sorted(kw))) >= N - 2


@pytest.mark.parametrize("dt", TYPES)
def test_list_ends(dt):
    """As many equal logits at the cut as the lists of long rows hold, and one more; counts up to and past those that
    are cut in a list."""
    V = 6000
    for n in (511, 512, 513, 700):
        z = torch.full((8, V), -4.0)
        z[:, 100:100 + n] = 1.0
        z[:, 3] = 2.0
        z[4:] += torch.rand(4, V, generator=torch.Generator().manual_seed(n)) * 2.0 ** -6
        z = z.to(dt).cuda()
        u = torch.tensor([0.0, 0.3, 0.7, 1 - 2.0 ** -24] * 2).cuda()
        for kw in (dict(top_k=n), dict(top_k=n // 2), dict(top_k=256), dict(top_k=257, top_p=0.5), dict(top_p=0.4),
                   dict(top_k=1), dict(temperature=0.0), dict(top_k=255, top_p=0.99, min_p=0.5)):
            say("sample, lists", n, dt, kw)
            check(reno.sample_symbols(z, u, **kw), draw(z, u, **kw), V, (n, dt, kw))


def test_long_offsets():
    """Rows whose offset passes 2^31 elements, the largest alphabet."""
    V = 1 << 20
    N = (1 << 31) // V + 3
    z = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    z[:, 11] = 30.0
    z[N - 1, 11] = 0.0
    z[N - 1, V - 1] = 30.0
    u = torch.full((N,), 0.5, device="cuda")
    say("sample, long", N, V)
    r = reno.sample_symbols(z, u)
    assert r.symbol[:-1].tolist() == [11] * (N - 1) and r.symbol[-1].item() == V - 1
    r = reno.sample_symbols(z[-2:], u[-2:], top_p=0.75)
    assert r.symbol.tolist() == [11, V - 1]
    z[-1] = 0.0
    r = reno.sample_symbols(z[-1:], u[-1:])
    assert r.symbol.item() == V // 2 and r.bits.item() == 20.0
    r = reno.sample_symbols(z[-1:], u[-1:], top_k=V // 4, top_p=0.5)
    assert r.symbol.item() == V // 16 and r.bits.item() == 17.0
    # the longest rows of 32 bits: the most turns of a wave
    z = torch.zeros(300, V, device="cuda")
    z[:, 0] = 1.0
    for rows in (1, 300):
        r = reno.sample_symbols(z[:rows], torch.full((rows,), 0.75, device="cuda"), top_p=0.5, top_k=V - 1)
        # weights e and V - 2 ones: half of them are the first and n ones, and u lies within the ones
        n = math.ceil(0.5 * (V - 2 + math.e) - math.e)
        W = n + math.e
        assert r.symbol.tolist() == [math.floor(0.75 * W - math.e) + 1] * rows
        assert r.bits[0].item() == pytest.approx(math.log2(W), abs=1e-6)


@pytest.mark.parametrize("V", [5, 270])
def test_rows_of_several_launches(V):
    """More rows than one launch takes: every row's own logits, settings and mask are found."""
    N = (1 << 21) + 37
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn(N, V, generator=g, device="cuda").to(torch.bfloat16)
    u = torch.rand(N, generator=g, device="cuda")
    T = 0.5 + torch.rand(N, generator=g, device="cuda")
    k = torch.randint(0, 9, (N,), generator=g, device="cuda").int()
    p = torch.rand(N, generator=g, device="cuda")
    least = torch.rand(N, generator=g, device="cuda") * 0.1
    allowed = torch.rand(N, V, generator=g, device="cuda") < 0.9
    say("sample, launches", N, V)
    r = reno.sample_symbols(z, u, T, k, p, least, allowed)
    for a, b in ((0, 50), ((1 << 21) - 20, N)):
        s = slice(a, b)
        part = reno.sample_symbols(z[s], u[s], T[s], k[s], p[s], least[s], allowed[s])
        assert torch.equal(r.symbol[s], part.symbol) and torch.equal(r.bits[s], part.bits)
        check(part, draw(z[s], u[s], T[s], k[s], p[s], least[s], allowed[s]), V, V)


def test_refusals():
    z, u = torch.zeros(4, 9, device="cuda"), torch.zeros(4, device="cuda")
    for bad in (dict(logits=z.cpu()), dict(logits=z.double()), dict(logits=z[0]), dict(u=u[:3]), dict(u=u.double()),
                dict(u=u.cpu()), dict(temperature=u[:3]), dict(temperature=u.double()), dict(top_k=u), dict(top_k=1.5),
                dict(top_k=-1), dict(top_k=1 << 31), dict(allowed=torch.ones(8, dtype=torch.bool, device="cuda")),
                dict(allowed=torch.ones(4, 9, device="cuda")), dict(allowed=torch.ones(1, 1, 9, device="cuda").bool())):
        with pytest.raises(ValueError):
            reno.sample_symbols(**{**dict(logits=z, u=u), **bad})
    for bad in (dict(temperature=-1.0), dict(temperature=math.nan), dict(top_p=1.5), dict(top_p=-0.1), dict(min_p=2.0)):
        with pytest.raises(reno.RenoError) as e:
            reno.sample_symbols(z, u, **bad)
        assert e.value.status == reno.RENO_E_INVALID


def test_capture_and_streams():
    z, u = make(100, 500, torch.float32, 3)
    big, ub = make(2, 60000, torch.bfloat16, 4)
    allowed = torch.arange(500, device="cuda") > 0
    want = [*reno.sample_symbols(z, u, top_p=0.8, allowed=allowed), *reno.sample_symbols(big, ub, top_k=40, top_p=0.9)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [*reno.sample_symbols(z, u, top_p=0.8, allowed=allowed), *reno.sample_symbols(big, ub, top_k=40, top_p=0.9)]
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(reno.sample_symbols(z, u, top_p=0.8, allowed=allowed).symbol, want[0])
    # another stream than the current one, its inputs freed right after the call
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a, b = z.clone(), u.clone()
    s.wait_stream(torch.cuda.current_stream())
    r = reno.sample_symbols(a, b, top_p=0.8, allowed=allowed, stream=s)
    del a, b
    torch.full_like(z, 7.0)
    s.synchronize()
    assert torch.equal(r.symbol, want[0]) and torch.equal(r.bits, want[1])


def test_frequencies():
    """Symbols of a uniform u come as often as their weights say: a binomial's deviation, 6 of them."""
    V, N = 37, 1 << 17
    z = torch.randn(V, generator=torch.Generator().manual_seed(1)).cuda()
    u = ((torch.arange(N) + 0.5) / N).cuda()
    r = reno.sample_symbols(z.expand(N, V), u)
    p = torch.softmax(z.double(), 0)
    n = torch.bincount(r.symbol.long(), minlength=V).double()
    assert bool(((n - p * N).abs() <= 1.0 + 1e-6 * N).all())   # evenly spaced u: off by one at either border
    assert torch.allclose(r.bits.double(), -torch.log2(p[r.symbol.long()]), atol=1e-6)


@pytest.mark.parametrize("which", [0, 1])
def test_a_frame_continued_by_draws(scan_cache, which):
    """A decoder that has the codes of a frame's coarse scales draws those of the next from the model's logits."""
    cfg = CONFIGS[which]
    B, b0 = cfg.bit_depth, cfg.min_bit_depth
    pts = scan_cache(which)
    w = reno.weights_to_device(gen_weights(cfg.channels, cfg.layers, seed=3, bias_std=0.1))
    enc = make_ctx(cfg_dict(cfg), len(pts))
    enc.set_weights(w)
    encode(enc, pts, B)
    codes = {b: enc.occupancy_codes(b).clone() for b in range(b0, B)}
    dec = make_ctx(cfg_dict(cfg), 8 * len(pts))
    dec.set_weights(w)
    dec.set_base(B, enc.coords(b0)[0].clone(), codes[b0])
    some = torch.arange(256, device="cuda") > 0          # a voxel has a child
    stop = b0 + 3
    for b in range(b0 + 1, stop + 1):
        dec.expand(b - 1, None if b - 1 == b0 else codes[b - 1])
        dec.predict_probs(b)
    logits = dec.predict_probs(stop, logits=True)
    N = logits.shape[0]
    u = torch.rand(N, generator=torch.Generator().manual_seed(9)).cuda()
    say("continue", cfg.name, N)
    r = reno.sample_symbols(logits, u, top_p=0.9, allowed=some)
    check(r, draw(logits, u, top_p=0.9, allowed=some), 256)
    assert bool((r.symbol >= 1).all())
    dec.expand(stop, r.symbol.to(torch.uint8))
    assert dec.num_voxels(stop + 1) == int(np.unpackbits(r.symbol.to(torch.uint8).cpu().numpy()).sum())
    enc.close()
    dec.close()
