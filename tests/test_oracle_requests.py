"""Pins of the oracle's definitions of sampling options and adapters
(oracle.requests): hand-worked rows, the definition said another way (token by
token, without sorting), and the law of the drawn tokens."""
import math

import numpy as np
import pytest

from oracle import requests as rq


def said_again(z, t, k, p, m):
    """The kept set token by token: rank = larger logits plus equal ones before."""
    z = [float(x) for x in z]
    el = [i for i, x in enumerate(z) if x == x and x > -math.inf]
    if not el:
        return set()
    top = max(z[i] for i in el)
    if top == math.inf or not t > 0:
        el = [i for i in el if z[i] == top]
    w = {i: 1.0 if z[i] == top else math.exp((z[i] - top) / t) for i in el}
    if not t > 0:
        return {min(el)}
    total, kept = math.fsum(w.values()), set()
    for i in el:
        ahead = [j for j in el if z[j] > z[i] or (z[j] == z[i] and j < i)]
        ok = (k <= 0 or len(ahead) < k) and (not p < 1 or math.fsum(w[j] for j in ahead) < p * total) and \
            (not m > 0 or w[i] >= min(m, 1.0))
        if ok or not ahead:
            kept.add(i)
    return kept


@pytest.mark.parametrize("seed", range(40))
def test_kept_sets(seed):
    r = np.random.default_rng(seed)
    z = r.normal(size=r.integers(1, 30)) * 2
    if seed % 3 == 0:
        z = np.round(z)
    if seed % 4 == 1:
        z[r.random(z.size) < 0.4] = -np.inf
    if seed % 5 == 2:
        z[r.random(z.size) < 0.3] = np.nan
    if seed % 7 == 3:
        z[r.integers(z.size)] = np.inf
    t, k, p, m = r.choice([0.0, 0.5, 1.0, 2.0]), int(r.choice([0, 1, 3, 100])), r.choice([1.0, 0.3, 0.9, 0.0]), r.choice([0.0, 0.2, 1.0])
    lw, keep, _ = rq.filter_row(z, t, k, p, m)
    assert set(np.flatnonzero(keep)) == said_again(z, t, k, p, m)
    assert np.all(np.isneginf(lw) == ~keep) or not t > 0 or np.isinf(z).any()


def test_rows_worked_by_hand():
    z = np.log([0.5, 0.25, 0.125, 0.125])
    for p, n in ((0.49, 1), (0.51, 2), (0.74, 2), (0.76, 3), (0.874, 3), (0.9, 4), (1.0, 4), (0.0, 1)):
        assert rq.filter_row(z, top_p=p)[1].sum() == n, p
    assert list(rq.filter_row(z, top_k=3)[1]) == [True, True, True, False]  # the tie's lower index
    assert list(rq.filter_row(z, min_p=0.4)[1]) == [True, True, False, False]
    lw, keep, _ = rq.filter_row(z, temperature=0.5)
    w = np.exp(lw)
    assert np.allclose(w / w.sum(), np.array([16, 4, 1, 1]) / 22)
    assert rq.draw_row(lw, keep, 0.0)[0] == 0 and rq.draw_row(lw, keep, 0.9999999)[0] == 3
    assert rq.draw_row(lw, keep, float(np.float32(16 / 22)) + 1e-4)[0] == 1
    assert rq.filter_row([-np.inf, np.nan])[1].sum() == 0 and rq.draw_row(np.full(2, -np.inf), np.zeros(2, bool), 0.5)[0] == -1


def test_draws_follow_the_filtered_law():
    r = np.random.default_rng(3)
    z = r.normal(size=12) * 1.5
    lw, keep, _ = rq.filter_row(z, 0.8, 8, 0.95, 0.02)
    p = np.where(keep, np.exp(lw), 0)
    p /= p.sum()
    n = 4000
    toks = [rq.draw_row(lw, keep, np.float32((i + 0.5) / n))[0] for i in range(n)]
    # an even grid of uniforms: each token's share within one step of its probability
    assert np.all(np.abs(np.bincount(toks, minlength=12) / n - p) <= 1.0 / n + 1e-6)


def test_adapters():
    r = np.random.default_rng(5)
    a, b, s = r.normal(size=(2, 6, 5)), r.normal(size=(2, 7, 3)), np.array([2.0, -1.0])
    x, y = r.normal(size=(3, 5)), r.normal(size=(3, 7))
    out = rq.lora(y, x, [1, -1, 0], a, b, s, [4, 3])
    assert np.array_equal(out[1], y[1])
    for t, i in ((0, 1), (2, 0)):
        full = np.zeros((7, 5))
        full[:4], full[4:] = b[i, :4] @ a[i, :3], b[i, 4:] @ a[i, 3:]
        assert np.allclose(out[t], y[t] + s[i] * (full @ x[t]))
