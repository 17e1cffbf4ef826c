"""The inner result A x between an adapter's two products: all of its fp32 bits
reach the second product, and its infinities stay infinities.

Tolerance: that of fp32 sums alone (test_gpu_lora), (d_in + rank + 8) 2^-24 of
the sum of absolute products and the output's rounding, also for bf16 weights,
without a share for the inner result.  d_in and rank are small, so that 16 bits
of it (2^-18 of a value) would not pass: with d_in 8 and rank 1 the bound is
17 * 2^-24, under 2^-19."""
import numpy as np
import pytest
import torch

from test_gpu_lora import apply, make

pytestmark = pytest.mark.gpu


def reference(c):
    x = c["x"].double().numpy() + (0 if c["x_lo"] is None else c["x_lo"].double().numpy())
    a, b, scale, y = (c[k].double().numpy() for k in ("a", "b", "scale", "y"))
    rank, ref, size = b.shape[2], y.copy(), np.zeros_like(y)
    for t, i in enumerate(c["ids"]):
        if not 0 <= i < a.shape[0]:
            continue
        o = 0
        for s, w in enumerate(c["segs"]):
            A, B = a[i, s * rank:(s + 1) * rank], b[i, o:o + w]
            ref[t, o:o + w] += scale[i] * (B @ (A @ x[t]))
            size[t, o:o + w] = abs(scale[i]) * (np.abs(B) @ (np.abs(A) @ np.abs(x[t])))
            o += w
    return ref, size


@pytest.mark.parametrize("T,rank,segs", [
    (40, 1, [640]), (40, 2, [300, 200]), (40, 8, [512]), (33, 40, [256]), (20, 70, [300]), (40, 128, [256]),      # 16-row tiles
    (4200, 1, [128]), (9000, 2, [130]), (6000, 8, [64, 64]), (2000, 33, [160]), (1100, 64, [192]), (700, 100, [300]), (600, 128, [256]),
])
@pytest.mark.parametrize("planes", [1, 2])
def test_all_bits_of_the_inner_result(T, rank, segs, planes):
    c = make(T, 8, segs, rank, 2, "bf16", "f32", planes, seed=T + rank)
    c["y"].zero_()  # nothing else is in the sums
    got = apply(c).double().numpy()
    ref, size = reference(c)
    tol = size * (8 + rank + 8) * 2.0 ** -24 + np.abs(ref) * 2.0 ** -23
    worst = np.max(np.abs(got - ref) / (tol + 1e-30))
    assert worst <= 1.0, worst


@pytest.mark.parametrize("T", [20, 4500])
@pytest.mark.parametrize("rank", [1, 5, 8, 40, 72])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_inner_results(T, rank, dtype):
    """One inner result beyond fp32's range, or next to it: the output is an
    infinity of the product's sign, or the number."""
    c = make(T, 24, [72, 40], rank, 2, dtype, "f32", ids=np.arange(T) % 3 - 1, seed=rank)
    c["a"][:, 1:rank] = 0.0
    c["a"][:, rank + 1:] = 0.0
    c["a"][:, [0, rank]] = 0.0
    c["a"][:, [0, rank], 0] = 3.0e38   # A x = 3e38 x[0] in the first of each segment's rows
    c["b"][c["b"] == 0] = 1.0
    c["x"][:, 0] = torch.tensor([2.0, -2.0, 1.125])[torch.arange(T) // 3 % 3].to(c["x"].dtype)
    b = c["b"][:, :, 0].double().numpy()
    scale = c["scale"].double().numpy()
    got = apply(c).double().numpy()
    for t in range(T):
        i = c["ids"][t]
        if i < 0:
            assert np.array_equal(got[t], c["y"][t].double().numpy())
            continue
        h = float(c["a"][i, 0, 0]) * float(c["x"][t, 0])
        ref = np.sign(h * b[i] * scale[i]) * np.inf if abs(h) > 3.4028235677973366e38 else h * b[i] * scale[i]
        if np.isfinite(ref[0]):
            # (B h itself may pass fp32's range before it is scaled)
            on = np.abs(h * b[i]) < 3.4e38
            assert np.all(np.abs(got[t][on] - ref[on]) <= np.abs(ref[on]) * (1 + rank + 8) * 2.0 ** -24 + 1e30)
        else:
            assert np.array_equal(got[t], ref), (t, i, got[t][:4], ref[:4])
