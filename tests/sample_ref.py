"""Symbols drawn from logits, from the definition in 64 bits on the CPU, row by row and without sorting tricks, with how
far each decision is from its border."""
import math

import numpy as np
import torch


def draw_row(z, u, T, k, p, least, allowed):
    """(symbol, bits, margin) of one row: margin is the smallest distance of a decision from its border, relative to
    the mass it is taken in."""
    if not (0 <= u < 1):
        return -1, 0.0, 1.0
    if not (0 <= T < math.inf) or math.isnan(p) or math.isnan(least):
        return -1, math.nan, 1.0
    z = z.astype(np.float64)
    there = np.ones(len(z), bool) if allowed is None else allowed.astype(bool)
    if np.isnan(z[there]).any() or (z[there] == np.inf).any():
        return -1, math.nan, 1.0
    there = there & (z > -np.inf)
    ids = np.flatnonzero(there)
    if len(ids) == 0:
        return -1, 0.0, 1.0
    order = ids[np.lexsort((ids, -z[ids]))]
    if T == 0:
        return int(order[0]), 0.0, 1.0
    w = np.exp((z[order] - z[order[0]]) / T)
    if k > 0:
        order, w = order[:k], w[:k]
    margin = 1.0
    if p < 1:
        sums = np.cumsum(w)
        target = p * math.fsum(w)
        n = int(np.searchsorted(sums, target))       # the first prefix that reaches it
        n = min(n, len(w) - 1)
        # a border that is hit exactly (equal weights) is no doubt: the sums are exact then
        gaps = np.abs(sums[max(n - 1, 0):n + 1] - target) / sums[-1]
        exact = bool((w == 1).all())
        margin = min([margin] + ([] if exact or target <= 0 else list(gaps)))
        order, w = order[:n + 1], w[:n + 1]
    least = min(least, 1.0)
    if least > 0:
        keep = w >= least
        keep[0] = True
        near = np.abs(w - least) / least
        margin = min(margin, near[near > 0].min(initial=1.0))
        order, w = order[keep], w[keep]
    back = np.argsort(order)
    order, w = order[back], w[back]
    sums = np.cumsum(w)
    total = math.fsum(w)
    at = int(np.searchsorted(sums, u * total, side="right"))
    at = min(at, len(w) - 1)
    if not (w == 1).all() and u > 0:
        margin = min(margin, np.abs(sums - u * total).min() / total)
    return int(order[at]), float(math.log2(total) - math.log2(w[at])) if w[at] > 0 else math.inf, float(margin)


def draw(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, allowed=None):
    n = logits.shape[0]

    def each(x):
        return x.cpu().double().tolist() if torch.is_tensor(x) else [x] * n

    z, uu = logits.float().cpu().numpy(), u.cpu().double().tolist()
    T, k, p, least = each(temperature), each(top_k), each(top_p), each(min_p)
    a = None if allowed is None else allowed.cpu().numpy()
    rows = [draw_row(z[i], uu[i], T[i], int(k[i]), p[i], least[i], None if a is None else a if a.ndim == 1 else a[i])
            for i in range(n)]
    return (np.array([r[0] for r in rows], np.int64), np.array([r[1] for r in rows]), np.array([r[2] for r in rows]))


def off(V):
    """How far a mass may be off, relative to itself.  Weights are counted in units of 2^-S of the largest, S = 51 up to
    V = 2048 and 62 - ceil(log2 V) above, each off by half of one (many equal weights by the same half), and by 2^-46
    of itself: V / 2 units, and a mass holds the largest weight."""
    S = min(51, 62 - math.ceil(math.log2(V)))
    return V * 2.0 ** -(S + 1) + 2.0 ** -46


def check(got, want, V, say=""):
    """got: Samples of V symbols; want: draw(...).  Equal symbols where a decision is not next to its border (a prefix
    and the mass that it is a share of may both be off), bits to their rounding; returns how many rows were compared."""
    symbol, bits = got.symbol.cpu().numpy(), got.bits.cpu().numpy().astype(np.float64)
    ws, wb, margin = want
    sure = margin > 2 * off(V)
    wrong = np.flatnonzero(sure & (symbol != ws))
    assert len(wrong) == 0, (say, "row", int(wrong[0]), "got", int(symbol[wrong[0]]), "want", int(ws[wrong[0]]),
                             "margin", float(margin[wrong[0]]), "of", len(wrong))
    nan = np.isnan(wb)
    assert (np.isnan(bits) == nan)[sure].all(), say
    # one rounding to fp32, the mass as bits, and the 64-bit sums and logarithms of both sides
    bound = 2.0 ** -24 * np.abs(wb) + off(V) / math.log(2) + 2.0 ** -46
    ok = np.abs(bits - wb) <= bound
    assert (ok | nan | ~sure).all(), (say, bits[~(ok | nan)][:4], wb[~(ok | nan)][:4])
    return int(sure.sum())
