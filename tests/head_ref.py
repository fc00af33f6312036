"""The head's training operators from their definitions in 64 bits, with a
bound for each output of how far 32-bit sums and the operand types' roundings
can take it.

With eps = 2^-24 (a rounding to fp32) and u the half step of the operand type:
  z     one rounding for each product kept to 2^-24 and each sum:
        dz = (C + 16) 2 eps (|h| |w| + |b|)  (2 eps a sum: the matrix units may cut off)
  t     z times a rounded constant: + 3 eps |t|
  lse2  as far off as the largest t, + the sum's roundings (at most 64 in a chain and
        V / 1024 of parts, 2 eps each) and 4 eps of the exponentials, over ln 2, + 4 eps |lse2|
  p     p (e^x - 1), x = ln 2 (dt + dlse2 + 2 eps |t - lse2|) + 4 eps
  dz    |g| (dp + 4 eps (p + q)) and its rounding to the operands' type, u |dz| (fp32: 2 eps)
  dh    the bound of dz through |w|, (V + 16) 2 eps |dz| |w| of the sums, u |dh| of the result
and dw, db likewise.  fp16 adds the spacing below its normal range.
"""
import math

import torch

EPS = 2.0 ** -24
LN2 = math.log(2.0)
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def targets_of(symbol, V):
    """Dense target distribution [N][V], rows taken, rows whose target is outside."""
    N = symbol.shape[0]
    q = torch.zeros(N, V, dtype=torch.float64, device=symbol.device)
    ok = (symbol >= 0) & (symbol < V)
    q[torch.nonzero(ok).flatten(), symbol[ok].long()] = 1.0
    return q, symbol >= 0, symbol >= V


def targets_of_top(index, logit, T, V):
    N, k = index.shape
    there = index >= 0
    x = torch.where(there, logit.double() / T, -math.inf)
    taken = there.any(1) & ((x > -math.inf) | x.isnan()).any(1)
    bad = (index >= V).any(1) | x.isnan().any(1) | (x == math.inf).any(1)
    e = torch.exp(x - x.amax(1, keepdim=True).nan_to_num(0.0, 0.0, 0.0))
    qe = torch.where(taken[:, None] & ~bad[:, None], e / e.sum(1, keepdim=True), 0.0).nan_to_num(0.0)
    q = torch.zeros(N, V, dtype=torch.float64, device=index.device)
    q.scatter_add_(1, index.long().clamp(0, V - 1), torch.where(there, qe, 0.0))
    return q, taken | bad, bad


def reference(h, w, b, q, taken, bad, g=None, T=1.0):
    """{name: (value, bound)} of bits, lse, dh, dw, db."""
    dt = h.dtype
    u = HALF_STEP[dt]
    N, C = h.shape
    V = w.shape[1]
    x = torch.where(taken[:, None], h.double(), 0.0)
    wd = w.double()
    bd = torch.zeros(V, dtype=torch.float64, device=w.device) if b is None else b.double()
    z = x @ wd + bd
    ez = (C + 16) * 2 * EPS * (x.abs() @ wd.abs() + bd.abs().nan_to_num(posinf=0.0))
    c = 1.0 / (T * LN2)
    t, et = z * c, ez * c
    et = et + 3 * EPS * t.abs().nan_to_num(posinf=0.0)
    lse2 = torch.logsumexp(z / T, 1) / LN2
    big = t.amax(1, keepdim=True).nan_to_num(0.0, 0.0, 0.0)
    near = torch.where(t > big - 60, et, 0.0).amax(1)
    el = near + ((64 + V / 1024 + 4) * 2 * EPS) / LN2 + 4 * EPS * lse2.abs()
    logp2 = t - lse2[:, None]
    p = torch.exp2(logp2)
    ex = LN2 * (et + el[:, None] + 2 * EPS * logp2.abs().nan_to_num(posinf=0.0)) + 4 * EPS
    ep = torch.where(p > 0, p * torch.expm1(ex), 0.0)      # logits far below the row's largest: exactly 0
    bits = torch.where(q > 0, q * (torch.where(q > 0, q, 1.0).log2() - logp2), 0.0).sum(1)
    k = (q > 0).sum(1)
    eb = (q * (et + el[:, None] + 8 * EPS * (1 + logp2.abs().nan_to_num(posinf=0.0)))).sum(1) * 1.01 + \
        (16 + k) * 2 * EPS * (q * logp2.abs()).nan_to_num(posinf=0.0).sum(1) + 16 * EPS * (1 + k)
    nan = torch.full_like(bits, math.nan)
    bits = torch.where(bad, nan, torch.where(taken, bits, 0.0))
    eb = torch.where(taken & ~bad, eb, 0.0)
    out = {"bits": (bits, eb),
           "lse": (torch.where(taken, lse2 * LN2, 0.0), torch.where(taken, el * LN2 + 2 * EPS * (lse2 * LN2).abs(), 0.0))}
    gd = torch.ones(N, dtype=torch.float64, device=h.device) if g is None else g.double()
    gd = torch.where(bad, nan, torch.where(taken, gd, 0.0))
    s = (gd * c)[:, None]
    dz = torch.where(taken[:, None], s * (p - q), 0.0)
    tiny = 2.0 ** -38 * s.abs().nan_to_num(0.0).max() if dt == torch.float16 else 0.0
    ez = torch.where(taken[:, None], s.abs() * (ep + 16 * EPS * (p + q)), 0.0) + max(u, 2 * EPS) * dz.abs() + tiny
    step = 2.0 ** -25 if dt == torch.float16 else 0.0     # half the spacing of fp16's smallest numbers
    ax, aw, ad = x.abs(), wd.abs(), dz.abs()

    def rounded(v, e):
        return v, e + u * (v.abs() + e) + step

    out["dh"] = rounded(dz @ wd.T, ez @ aw.T + (V + 16) * 2 * EPS * (ad @ aw.T) * 1.01)
    out["dw"] = rounded(x.T @ dz, ax.T @ ez + (N + 16) * 2 * EPS * (ax.T @ ad) * 1.01)
    out["db"] = rounded(dz.sum(0), ez.sum(0) + (N + 16) * 2 * EPS * ad.sum(0))
    return out


def check(name, got, value, bound):
    got = got.double().cpu()
    value, bound = value.cpu(), bound.cpu()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    same = (got == value) | (got.isnan() & value.isnan())
    off = (got - value).abs()
    ok = same | (off <= bound)
    if not bool(ok.all()):
        at = torch.nonzero(~ok)[0].tolist()
        i = tuple(at)
        raise AssertionError(f"{name}: {int((~ok).sum())} of {ok.numel()} outside, first at {at}: got {got[i].item()!r}, "
                             f"want {value[i].item()!r} within {bound[i].item():.3g}")
