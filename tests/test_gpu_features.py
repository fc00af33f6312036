"""Features of every kind of context: the full predictor, its wide and 5x5x5
layers, the two-stage head and the plain model of one to four layers.  The head
of the weights, applied to them in 64 bits, gives the logits that the model's
own kernels gave; and a two-stage head takes a training step from them."""
import math

import numpy as np
import pytest
import torch

import paper_2503_12382_amd as reno
from gpu_helpers import say, to_dev
from head_ref import check, reference, targets_of
from synth import gen_weights

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def cloud(seed, n, B):
    rs = np.random.default_rng(seed)
    xyz = np.concatenate([rs.integers(0, 1 << B, size=(n // 4, 3)),
                          rs.integers(0, 1 << (B - 2), size=(n - n // 4, 3)) + (1 << (B - 3))])
    return (-10.0 + (xyz + 0.5) * (20.0 / (1 << B))).astype(np.float32)


def within(logits, h, w, b, C):
    """A product to 2^-20 of the sum of its absolute values, and its roundings (RENO_PREC_FP32)."""
    z = h.double() @ w.double() + b.double()
    size = h.double().abs() @ w.double().abs() + b.double().abs()
    assert bool(((logits.double() - z).abs() <= (2.0 ** -20 + (C + 16) * 2 * EPS) * size).all())


# C, layers, full predictor, kernel size, two-stage
KINDS = [(16, 1, False, 3, False), (32, 3, False, 3, False), (32, 2, False, 3, True), (16, 4, False, 3, True),
         (16, 2, True, 3, False), (32, 2, True, 3, True), (64, 2, True, 3, False), (32, 2, True, 5, False),
         (128, 2, True, 5, True), (128, 2, True, 3, False)]


@pytest.mark.parametrize("C,L,top,ks,two", KINDS)
def test_features_give_the_logits(C, L, top, ks, two):
    B, b0 = 7, 3
    pts = cloud(C + ks + L, 1500, B)
    w = reno.weights_to_device(gen_weights(C, L, seed=50 + C + ks + L, bias_std=0.1, two_stage=two, top=top, kernel_size=ks))
    say("features C", C, "layers", L, "full", top, "k", ks, "two-stage", two)
    ctx = reno.Context(len(pts), B, b0, 10.0, C, L, two_stage=two, top=top, kernel_size=ks)
    ctx.set_weights(w)
    ctx.build_pyramid(to_dev(pts), B)
    logits = ctx.predict_probs(reno.RENO_ALL_SCALES, logits=True)
    h = ctx.features(reno.RENO_ALL_SCALES)
    assert h.shape == (logits.shape[0], C) and bool(h.isfinite().all()) and bool(h.any())
    codes = torch.cat([ctx.occupancy_codes(b) for b in range(b0 + 1, B)]).long()
    heads = ([(h, w["head1_w"], w["head1_b"], logits[:, :16]),
              (h + w["emb_s1"][codes & 15], w["head2_w"], w["head2_b"], logits[:, 16:])]
             if two else [(h, w["head_w"], w["head_b"], logits)])
    for x, hw, hb, z in heads:
        within(z, x, hw, hb, C)
    # one scale at a time, as the decoder goes, leaves the same
    off = 0
    for b in range(b0 + 1, B):
        n = ctx.num_voxels(b)
        assert torch.equal(ctx.features(b), h[off:off + n])
        ctx.predict_probs(b)
        assert torch.equal(ctx.features(b), h[off:off + n])
        off += n
    assert off == h.shape[0]
    # and what follows a prediction does not touch them
    ctx.code_length(reno.RENO_ALL_SCALES)
    if two:
        ctx.predict_second(B - 1)
    ctx.symbol_intervals(reno.RENO_ALL_SCALES)
    assert torch.equal(ctx.features(reno.RENO_ALL_SCALES), h)
    # a new frame has none
    ctx.build_pyramid(to_dev(pts[:700]), B)
    with pytest.raises(reno.RenoError) as e:
        ctx.features(B - 1)
    assert e.value.status == reno.RENO_E_STATE
    ctx.close()


@pytest.mark.parametrize("top", [False, True])
def test_features_do_not_depend_on_the_head(top):
    """What a head that starts from zero is trained on: the features under any head without zero rows."""
    C, B, b0 = 32, 7, 3
    pts = cloud(3, 1200, B)
    w = gen_weights(C, 2, seed=9, bias_std=0.1, top=top)
    say("features under several heads", top)
    ctx = reno.Context(len(pts), B, b0, 10.0, C, 2, top=top)
    ctx.build_pyramid(to_dev(pts), B)
    seen = []
    # (with the full predictor, whose layers read every channel, zero rows are no loss)
    for scale in (1.0, 2.0 ** -30, -3.0) + ((0.0,) if top else ()):
        ctx.set_weights(reno.weights_to_device(dict(w, head_w=w["head_w"] * np.float32(scale))))
        ctx.predict_probs(reno.RENO_ALL_SCALES)
        seen.append(ctx.features(reno.RENO_ALL_SCALES))
    # the head's balance, a power of two, does not change the sums that it multiplies
    for h in seen[1:]:
        assert bool(((h - seen[0]).abs() <= 2.0 ** -18 * seen[0].abs().amax()).all())
    ctx.close()


def test_a_training_step_of_a_two_stage_head():
    """Both 16-symbol heads from the features, the second from h + Emb(S1); the codec's own bits are theirs."""
    C, B, b0 = 32, 7, 3
    pts = cloud(5, 1500, B)
    w = reno.weights_to_device(gen_weights(C, 2, seed=31, bias_std=0.1, two_stage=True))
    say("a training step of a two-stage head")
    ctx = reno.Context(len(pts), B, b0, 10.0, C, 2, two_stage=True)
    ctx.set_weights(w)
    ctx.build_pyramid(to_dev(pts), B)
    ctx.predict_probs(reno.RENO_ALL_SCALES)
    h = ctx.features(reno.RENO_ALL_SCALES)
    per, _ = ctx.code_length(reno.RENO_ALL_SCALES)
    codes = torch.cat([ctx.occupancy_codes(b) for b in range(b0 + 1, B)]).int()
    s1, s2 = codes & 15, codes >> 4
    x2 = h + w["emb_s1"][s1.long()]
    N = h.shape[0]
    g = torch.full((N,), 1.0 / N, device="cuda")
    r1 = reno.head_code_length(h, w["head1_w"], w["head1_b"], s1, row_weight=g, grad=True)
    r2 = reno.head_code_length(x2, w["head2_w"], w["head2_b"], s2, row_weight=g, grad=True)
    for r, x, a, b, s in ((r1, h, "head1_w", "head1_b", s1), (r2, x2, "head2_w", "head2_b", s2)):
        ref = reference(x, w[a], w[b], *targets_of(s, 16), g)
        for name in ("bits", "lse", "dh", "dw", "db"):
            check(name, getattr(r, name), *ref[name])
    size = torch.cat([h.double().abs() @ w["head1_w"].double().abs(), x2.double().abs() @ w["head2_w"].double().abs()], 1)
    assert bool(((r1.bits.double() + r2.bits.double() - per.double()).abs()
                 <= 8 * (2.0 ** -20 + (C + 16) * 2 * EPS) * size.amax(1) / math.log(2.0) + 1e-5).all())
    # the gradients against central differences of the loss in 64 bits, along themselves: 1e-4 squared of the third
    # derivative, and fp32 gradients
    grads = {"head1_w": r1.dw, "head1_b": r1.db, "head2_w": r2.dw, "head2_b": r2.db}
    square = sum(float((d.double() ** 2).sum()) for d in grads.values())

    def loss(step):
        out = 0.0
        for x, a, b, s in ((h, "head1_w", "head1_b", s1), (x2, "head2_w", "head2_b", s2)):
            z = x.double() @ (w[a].double() + step * grads[a]) + w[b].double() + step * grads[b]
            out += float((torch.logsumexp(z, 1) - z.gather(1, s.long()[:, None])[:, 0]).mean()) / math.log(2.0)
        return out
    assert abs((loss(1e-4) - loss(-1e-4)) / 2e-4 - square) <= 1e-5 * square
    ctx.close()
