"""Definitions in 64 bits of what a request brings of its own: its sampling
options (temperature, top-k, top-p, min-p) and its low-rank adapter.  Plain
numpy, one row at a time; test infrastructure like the rest of the oracle."""
from __future__ import annotations

import numpy as np


def filter_row(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(log-weights, kept, gap) of one row of logits.

    log-weights: (z - m) / T, float64, -inf where not kept; kept: bool;
    gap: how near the nearest sum that decided something came to its border,
    relative to the smallest weight that it decided about (inf: none did)."""
    z = np.asarray(z, np.float64)
    V = z.size
    none = np.full(V, -np.inf), np.zeros(V, bool), np.inf
    with np.errstate(invalid="ignore"):
        eligible = z > -np.inf
    if not eligible.any():
        return none
    m = z[eligible].max()
    if m == np.inf:
        eligible = z == m
    t, p, mp = float(temperature), float(top_p), float(min_p)
    greedy = not t > 0.0
    if greedy:
        eligible = z == m
    zz = np.where(eligible, z, -np.inf)
    order = np.argsort(-zz, kind="stable")[:int(eligible.sum())]
    with np.errstate(invalid="ignore", over="ignore"):
        lw = np.where(zz == m, 0.0, 0.0 if greedy else (zz - m) / (t if not greedy else 1.0))
    lw = np.where(eligible, lw, -np.inf)
    w = np.exp(lw[order].astype(np.longdouble))
    n, gap = order.size, np.inf
    if greedy:
        n = 1
    if top_k > 0:
        n = min(n, int(top_k))
    if p < 1.0:
        before = np.concatenate(([0.0], np.cumsum(w)[:-1])).astype(np.longdouble)
        P = np.longdouble(p) * w.sum()
        c = int(np.searchsorted(before, P, side="left"))
        near = np.abs(before - P)
        # (a sum equal to its border is as exact as the weights are: powers of two)
        near = np.where((near == 0) | (w == 0), np.inf, near)
        gap = float(np.min(near / np.where(w == 0, 1, w))) if P > 0 else np.inf
        n = min(n, c)
    if mp > 0.0:
        # (by logarithms: exp(-1e-30) rounds to 1, which a smaller logit's weight never is)
        n = min(n, int(np.count_nonzero(lw[order] >= np.log(min(mp, 1.0)))))
    n = max(n, 1)
    kept = np.zeros(V, bool)
    kept[order[:n]] = True
    return np.where(kept, lw, -np.inf), kept, gap


def draw_row(lw, kept, u):
    """(token, probability, gap) of the first kept token whose running sum of
    weights exceeds u times their sum; gap: distance of u from the borders of
    the drawn token's interval, over its probability."""
    if not kept.any():
        return -1, 0.0, np.inf
    u = np.float32(u)
    u = min(max(float(u), 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    w = np.where(kept, np.exp(lw.astype(np.longdouble)), 0)
    cum = np.cumsum(w)
    x = np.longdouble(u) * cum[-1]
    k = int(np.searchsorted(cum, x, side="right"))
    lo = cum[k] - w[k]
    near = min(cum[k] - x, x - lo if x > lo else np.inf)
    return k, float(w[k] / cum[-1]), float(near / w[k])


def lora(y, x, ids, a, b, scale, segs):
    """y + scale[i] B_i (A_i x) row by row, i = ids[t]; float64."""
    out = np.array(y, np.float64)
    rank = b.shape[2]
    for t, i in enumerate(ids):
        if not 0 <= i < a.shape[0]:
            continue
        c = 0
        for s, width in enumerate(segs):
            h = a[i, s * rank:(s + 1) * rank].astype(np.float64) @ x[t].astype(np.float64)
            out[t, c:c + width] += float(scale[i]) * (b[i, c:c + width].astype(np.float64) @ h)
            c += width
    return out
