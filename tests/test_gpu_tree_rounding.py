"""Tree attention over scores that are exact in fp32 but large: what rounding the
running maxima does to the weights (sd_tree_attention against oracle.trees).

A score is B + x f, B a power of two and x f on fp32's grid there, so it has no error.
With n keys and U = 2^-24 that leaves, relative to the sum of weights * |value|:
exponents of up to D = 64 (what weighs less than 2^-64 does not count), rounded three times
in numerator and denominator; the exponentials and the products of a rescaling
or a merge, 2^-22 for each of at most one per block of 32 keys and 8 more; 2^-17 of a
weight that its two bf16 planes leave out; two sums over n keys; and the output's
rounding.  Maxima kept as rounded products, with differences taken of the
unrounded ones, were off by 2^-5 in an exponent at B = 2^19: 2 %."""
import numpy as np
import pytest
import torch

from oracle import trees
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def plant(c, B, step, seed):
    """Rows with factors 1 and 1/8; maxima that grow from block to block by 12 steps and start again every ten
    blocks, a few steps of noise on top."""
    r = np.random.default_rng(seed)
    hd = c.hd
    q = np.zeros((c.T, c.hq, hd), np.float32)
    q[:, :, 0] = 1.0
    q[:, :, 1] = np.where(r.random((c.T, c.hq)) < 0.3, 1.0, 0.125)
    c.q = torch.from_numpy(q).to(c.q.dtype)
    if c.q_lo is not None:
        c.q_lo.zero_()
    c.pool[:, :, 0] = 0
    for b in range(len(c.prefix)):
        for x in range(int(c.prefix[b]) + int(c.off[b + 1] - c.off[b])):
            page, row = int(c.table[b, x // 16]), x % 16
            c.pool[:, page, 0, :, row * hd] = B
            c.pool[:, page, 0, :, row * hd + 1] = step * (12 * (x // 32 % 10) + 0.5 * int(r.integers(0, 9)))


def check(c, label, scale, n):
    torch.cuda.synchronize()
    q = c.q.double().numpy()
    ref, size, _ = trees.tree_attention(c.pool.double().numpy(), c.layer, c.off, c.prefix, c.table, c.parent, q, scale, c.hkv,
                                        c.max_slots)
    got = c.out.double().cpu().numpy()
    if c.out_lo is not None:
        got = got + c.out_lo.double().cpu().numpy()
    step = {"f32": 2.0 ** -24, "bf16": 2.0 ** -16 if c.planes == 2 else 2.0 ** -8}[c.dtype]
    rel = 2 * 3 * 64 * U + 2 * (n / 32 + 8) * 2.0 ** -22 + (2.0 ** -17 if c.dtype == "bf16" else 0.0) + 2 * n * U
    off = np.abs(got - ref) / (rel * size + step * np.abs(ref))
    print(f"{label}: worst {off.max():.3f} of the tolerance, {(np.abs(got - ref) / size).max():.2e} of the values", flush=True)
    assert off.max() <= 1.0, f"{label}: {off.max()} times the tolerance"


USERS = {
    "rescaled": ([(310 + i % 7, 1 + i % 3) for i in range(260)], 8),  # several blocks a workgroup, few rows
    "wide rows": ([(310 + i % 7, 12) for i in range(90)], 8),          # more than 64 rows
    "widest": ([(300, 20), (350, 17), (290, 18)] * 8, 10),             # more than 128 rows
    "parts": ([(1900, 3)], 8),                                         # a block a workgroup, merged
    "parts of wide rows": ([(1500, 13)], 8),
}


@pytest.mark.parametrize("where", USERS)
@pytest.mark.parametrize("B,step,scale", [(2.0 ** 10, 1.0, 0.75), (2.0 ** 19, 1.0, 0.75), (2.0 ** 21, 4.0, 0.6875), (2.0 ** 23, 16.0, 0.6875),
                                          (-(2.0 ** 19), 1.0, 0.75)])
def test_large_exact_scores(where, B, step, scale):
    users, G = USERS[where]
    c = Case(users, "bf16", 64, 1, G, kind="chain", planes=2, seed=31, layers=1, layer=0)
    plant(c, B, step, 32)
    c.to_gpu().call(scale=scale)
    check(c, f"{where} {B}", scale, max(p + n for p, n in users))


@pytest.mark.parametrize("hd", [128])
def test_large_exact_scores_of_larger_heads(hd):
    users, G = USERS["rescaled"]
    c = Case(users[:150], "bf16", hd, 2, G, kind="chain", planes=1, seed=33, layers=1, layer=0)
    c.planes, c.q_lo = 2, torch.zeros_like(c.q)
    plant(c, 2.0 ** 19, 1.0, 34)
    c.to_gpu().call(scale=0.75)
    check(c, "hd 128", 0.75, 330)


def test_large_exact_scores_fp32():
    c = Case([(310, 3), (1900, 2)], "f32", 64, 1, 4, kind="chain", seed=35, layers=1, layer=0)
    plant(c, 2.0 ** 19, 1.0, 36)
    c.to_gpu().call(scale=0.5)  # (a power of two: the scaled score is exact too)
    check(c, "fp32", 0.5, 1902)
