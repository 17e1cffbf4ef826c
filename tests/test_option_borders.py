"""The inputs of test_gpu_filter's exact comparisons stay away from the borders
where a rounded sum could decide otherwise than an exact one.  CPU only.

What a sum of the kernels is off by, in weights of the row's largest token: a
weight is rounded to 30 bits (half a step: 2^-31 of it) and to a multiple of
2^-37 (half a step: 2^-38), both with either sign, so a sum over the N tokens
that are in it is off by about 2^-31 sqrt(sum w^2) + 2^-38 sqrt(N), its merges
in 64-bit floating point by far less.  Four times that is asked of the distance
between each border -- top_p's, in the sums of all tokens, and the drawn
uniform's, in those of the kept ones -- and the sums next to it.  min_p
compares one logarithm, to 2^-50 of it.  (Sums equal to their border are left
out: they are sums of powers of two, exact on both sides.)"""
import numpy as np
import pytest

import test_gpu_filter as cases
from oracle import requests as rq


def distances(z, t, k, p, m, u):
    """Distances of top_p's border and of u's over the error of a sum, and of min_p's; infinite where there is none."""
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore"):
        z = np.where(z > -np.inf, z, -np.inf)
    top = z.max()
    if not np.isfinite(top) or not t > 0:
        return np.inf, np.inf, np.inf
    y = np.sort(z[z > -np.inf])[::-1].astype(np.longdouble)
    y = (y - top) / np.longdouble(t)
    w = np.exp(y)

    def error(w):
        return 2.0 ** -31 * float(np.sqrt((w * w).sum())) + 2.0 ** -38 * np.sqrt(w.size)

    def nearest(sums, border):
        d = np.abs(sums - border)
        d = d[d > 0]
        return float(d.min()) if d.size else np.inf

    dp = nearest(np.concatenate(([0], np.cumsum(w)[:-1])), np.longdouble(p) * w.sum()) if 0 < p < 1 else np.inf
    dm = nearest(y, np.log(np.longdouble(m))) if 0 < m < 1 else np.inf
    lw, keep, _ = rq.filter_row(z, t, k, p, m)
    u = min(max(float(u), 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    wk = np.exp(lw[keep].astype(np.longdouble))
    du = nearest(np.cumsum(wk), np.longdouble(u) * wk.sum()) if u > 0 else np.inf
    return dp / error(w), du / error(wk), dm


def check(host, t, k, p, m, u):
    for i in range(host.shape[0]):
        dp, du, dm = distances(host[i], t[i], k[i], p[i], m[i], u[i])
        assert dp > 4 and du > 4 and dm > 2.0 ** -40, (i, dp, du, dm)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", [k for k in cases.KINDS if k not in ("wide", "lowest")])
def test_kinds_of_rows(kind, dtype):
    check(cases.values(kind, 12, 5003, dtype, 5)[1], *cases.options(12, 7), cases.uniforms(12, 9))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_row_lengths(dtype):
    for V in (2, 3, 63, 64, 65, 255, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 8193, 32003):
        check(cases.values("normal", 7, V, dtype, V)[1], *cases.options(7, V), cases.uniforms(7, V))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["normal", "coarse", "flat", "constant", "masked", "two"])
def test_large_vocabulary(kind, dtype):
    check(cases.values(kind, 8, 151936, dtype, 51)[1], *cases.options(8, 53), cases.uniforms(8, 55))


def test_many_rows():
    check(cases.values("normal", 1100, 515, "f32", 71)[1], *cases.options(1100, 73), cases.uniforms(1100, 75))
