"""Filtered sampling and filtered logits (sd_sample_filtered, sd_filter_logits)
against their 64-bit definition (oracle.requests): kept sets and tokens are
equal, probabilities and log-weights within their last rounding.

Tolerances: log-weights and probabilities are computed in 64 bits and rounded
once, so they are off by at most half a step of fp32 (2^-24 relative) plus the
64-bit error, for which the same again is ample.  Whole results have no
tolerance; the oracle says how near a border each came, and the seeded inputs
here all stay further off than the 2^-40 of the kernels' fixed-point sums."""
import numpy as np
import pytest
import torch

from oracle import requests as rq
from paper_2604_20919_amd import sdverify as sv

pytestmark = pytest.mark.gpu

LOWEST = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def values(kind, n, V, dtype, seed):
    """n rows of V logits of one kind, float32 values that dtype holds exactly."""
    r = np.random.default_rng(seed)
    z = (r.standard_normal((n, V)) * r.uniform(0.5, 4.0, (n, 1))).astype(np.float32)
    if kind == "constant":
        z[:] = r.standard_normal((n, 1))
    elif kind == "two":
        z = np.where(r.random((n, V)) < 0.3, np.float32(1.5), np.float32(-0.25))
    elif kind == "coarse":  # many ties
        z = np.round(z * 2) / 2
    elif kind == "flat":
        z *= 0.01
    elif kind == "masked":
        z = np.where(r.random((n, V)) < 0.9, np.float32(-np.inf), z)
        z[0] = -np.inf
    elif kind == "lowest":  # masked by the type's lowest value instead
        z = np.where(r.random((n, V)) < 0.9, np.float32(LOWEST[dtype]), z)
        z[0] = LOWEST[dtype]
    elif kind == "nan":
        z = np.where(r.random((n, V)) < 0.3, np.float32(np.nan), z)
        z[0] = np.nan
    elif kind == "inf":
        z = np.where(r.random((n, V)) < 0.02, np.float32(np.inf), z)
        z[:, V // 2] = np.inf
    elif kind == "zeros":  # both zeros and the numbers next to them
        z = r.choice(np.array([0.0, -0.0, 1e-45, -1e-45, 1e-38, -1e-38], np.float32), (n, V))
    elif kind == "wide":
        z = (z * 1e37).astype(np.float32)
    t = torch.from_numpy(np.ascontiguousarray(z, np.float32)).to(DT[dtype])
    return t, t.float().numpy()


def options(n, seed, which="mixed"):
    r = np.random.default_rng(seed + 1000)
    t = r.choice([0.0, 0.3, 0.7, 1.0, 1.6], n).astype(np.float32)
    k = r.choice([0, 0, 1, 2, 7, 50, 1000], n).astype(np.int32)
    p = r.choice([1.0, 1.0, 0.1, 0.5, 0.9, 0.97], n).astype(np.float32)
    m = r.choice([0.0, 0.0, 0.02, 0.3], n).astype(np.float32)
    if which == "odd":  # every value means something
        t = r.choice(np.array([-1.0, np.nan, np.inf, 1e-30, 1e30, 0.5], np.float32), n)
        k = r.choice([-5, 1 << 30, 3], n).astype(np.int32)
        p = r.choice(np.array([-1.0, 0.0, np.nan, 2.0, np.inf, 0.75], np.float32), n)
        m = r.choice(np.array([-1.0, np.nan, 1.0, 3.0, 0.25, 1e-30], np.float32), n)
    return t, k, p, m


def uniforms(n, seed):
    u = np.random.default_rng(seed + 2000).random(n).astype(np.float32)
    special = np.array([0.0, 1.0 - 2.0 ** -24, 1.0, np.nan, -1.0, 2.0], np.float32)
    u[:min(n, special.size)] = special[:n] if n > 1 else u[:1]
    return u


def padded(t, pad, offset=0):
    """t in a wider buffer (rows V + pad apart, the first `offset` elements in); the rest is NaN."""
    n, V = t.shape
    buf = torch.full((n * (V + pad) + offset,), float("nan"), dtype=t.dtype, device="cuda")
    view = buf[offset:].as_strided((n, V), (V + pad, 1), offset)
    view.copy_(t)
    return view


def check(z, host, t, k, p, m, u, stream=None, workspace=None, near=False):
    """Both calls on device rows z (host: their values), against the oracle.

    near: rows with weights so small that they vanish beside the largest, drawn
    from at u = 0 too.  A weight is a multiple of 2^-37 of 2^G, G at most two
    above the largest's logarithm: it is off by 2^-36 of the largest at most, and
    a running sum by that times the number kept.  The token drawn is one whose
    interval u comes that near to."""
    n, V = host.shape
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    kept, kept2 = torch.full_like(token, -7), torch.full_like(token, -7)
    prob = torch.full((n,), -7.0, device="cuda")
    out = torch.full((n, V + 3), 7.0, device="cuda")
    ws = workspace if workspace is not None else torch.empty(sv.sd_filter_query_size(n, V), dtype=torch.uint8, device="cuda")
    o = dict(temperature=dev(t), top_k=dev(k), top_p=dev(p), min_p=dev(m))
    ud = dev(u)
    torch.cuda.synchronize()
    sv.sd_sample_filtered(z, ud, token, ws, prob=prob, kept=kept, stream=stream, **o)
    sv.sd_filter_logits(z, out[:, :V], ws, kept=kept2, stream=stream, **o)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    assert np.all(got[:, V:] == 7.0)
    token, kept, kept2, prob = (a.cpu().numpy() for a in (token, kept, kept2, prob))
    for i in range(n):
        lw, keep, gap = rq.filter_row(host[i], 1.0 if t is None else t[i], 0 if k is None else k[i],
                                      1.0 if p is None else p[i], 0.0 if m is None else m[i])
        tok, pr, gap2 = rq.draw_row(lw, keep, u[i])
        where = f"row {i}: T {t is not None and t[i]} k {k is not None and k[i]} p {p is not None and p[i]} " \
                f"min_p {m is not None and m[i]} u {u[i]} gaps {gap:.2e} {gap2:.2e}"
        assert kept[i] == keep.sum(), (where, kept[i], keep.sum())
        assert kept2[i] == kept[i], where
        assert np.array_equal(got[i, :V] > -np.inf, keep & (lw.astype(np.float32) > -np.inf)), where
        on = got[i, :V] > -np.inf
        ref = lw[on]
        assert np.all(np.abs(got[i, :V][on] - ref) <= 2 * 2.0 ** -24 * np.abs(ref) + 2.0 ** -149), where
        if near and token[i] != tok:
            w = np.exp(lw.astype(np.longdouble))
            cum = np.cumsum(w)
            x, eps = min(max(float(np.nan_to_num(u[i])), 0.0), 1.0 - 2.0 ** -24) * cum[-1], keep.sum() * 2.0 ** -36
            tok, pr = token[i], float(w[token[i]] / cum[-1])
            assert keep[tok] and cum[tok] - w[tok] - eps <= x <= cum[tok] + eps, where
        assert token[i] == tok, (where, token[i], tok)
        assert abs(prob[i] - pr) <= 2 * 2.0 ** -24 * pr, (where, prob[i], pr)


KINDS = ["normal", "constant", "two", "coarse", "flat", "masked", "lowest", "nan", "inf", "zeros", "wide"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_kinds_of_rows(kind, dtype):
    n, V = 12, 5003
    t, host = values(kind, n, V, dtype, 5)
    check(padded(t, 5), host, *options(n, 7), uniforms(n, 9))


@pytest.mark.parametrize("kind", ["normal", "coarse", "masked", "inf", "zeros"])
def test_every_option_value_has_a_meaning(kind):
    n, V = 40, 700
    t, host = values(kind, n, V, "f32", 15)
    check(t.cuda(), host, *options(n, 17, "odd"), uniforms(n, 19))


@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 255, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 8193, 32003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_row_lengths(V, dtype):
    n = 7
    t, host = values("normal", n, V, dtype, V)
    check(t.cuda(), host, *options(n, V), uniforms(n, V))


@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (2, 2), (3, 3), (4, 0), (61, 5), (64, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignments(pad, offset, dtype):
    n, V = 5, 2050
    t, host = values("normal", n, V, dtype, 31 + pad)
    check(padded(t, pad, offset), host, *options(n, 33 + pad), uniforms(n, 35))


@pytest.mark.parametrize("off", range(4))
def test_options_that_are_not_given(off):
    n, V = 9, 3001
    t, host = values("normal", n, V, "f32", 41)
    o = list(options(n, 43))
    o[off] = None
    check(t.cuda(), host, *o, uniforms(n, 45))
    o = [None] * 4
    check(t.cuda(), host, *o, uniforms(n, 47))


@pytest.mark.parametrize("kind", ["masked", "lowest", "nan", "inf", "wide", "coarse"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_stretches_without_a_token(kind, dtype):
    """All but a few short stretches of a long row masked: whole parts of it
    hold nothing but -inf or the type's lowest value."""
    n, V = 10, 40000
    t, host = values(kind, n, V, dtype, 57)
    t = t.clone()
    low = LOWEST[dtype] if kind in ("lowest", "wide") else float("-inf")
    for a, b in ((0, 8000), (8300, 24500), (24600, 39990)):
        t[:, a:b] = low
    check(t.cuda(), t.float().numpy(), *options(n, 58), uniforms(n, 59))
    check(t.cuda(), t.float().numpy(), None, None, None, None, uniforms(n, 60))


@pytest.mark.parametrize("kind", ["normal", "coarse", "flat", "constant", "masked", "two"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_vocabulary(kind, dtype):
    n, V = 8, 151936
    t, host = values(kind, n, V, dtype, 51)
    check(t.cuda(), host, *options(n, 53), uniforms(n, 55))


@pytest.mark.parametrize("V,dtype", [(9001, "f32"), (40000, "bf16"), (151936, "f32")])
@pytest.mark.parametrize("kind", ["normal", "coarse", "masked"])
def test_low_temperatures(V, dtype, kind):
    """Prefixes that end far below the largest weight."""
    n = 16
    t, host = values(kind, n, V, dtype, 91)
    T = np.array([0.61, 0.59, 0.3, 0.29, 0.15, 0.1, 0.05, 0.02, 0.01, 1e-3, 3e-4, 1e-4, 1e-5, 1e-8, 0.2, 0.1], np.float32)
    k = np.array([50, 1000, 50, 2000, 50, 1000, 100, 64, 5, 1000, 50, 700, 50, 50, 0, 0], np.int32)
    p = np.array([1.0, 0.999, 1.0, 1.0] * 4, np.float32)
    m = np.zeros(n, np.float32)
    m[14:] = 1e-20, 1e-30
    check(t.cuda(), host, T, k, p, m, uniforms(n, 93), near=True)
    check(t.cuda(), host, T, k, None, m, uniforms(n, 95), near=True)


@pytest.mark.parametrize("big", [-1e9, 1e10, 3e11, -7.5e7, 1e6])
def test_masked_beside_logits_far_from_zero(big):
    """Logits so far from zero that one step of fp32 is many octaves of weight,
    with -inf and not-a-numbers beside them: those weigh nothing."""
    n, V = 12, 9001
    r = np.random.default_rng(81)
    z = np.full((n, V), -np.inf, np.float32)
    at = r.integers(0, V, (n, 40))
    for i in range(n):
        z[i, at[i]] = np.nextafter(np.float32(big), np.float32(-np.inf if i % 2 else big))
        z[i, at[i, :3]] = np.float32(big)
        z[i, at[i, 20:25]] = np.nan
    t, host = torch.from_numpy(z), z
    T = np.array([1.0, 0.5, 0.3, 2.0] * 3, np.float32)
    check(t.cuda(), host, T, None, None, None, uniforms(n, 83), near=True)
    check(t.cuda(), host, T, np.array([0, 2, 5, 100] * 3, np.int32), np.array([0.9, 0.5, 1.0, 0.999] * 3, np.float32),
          np.array([0.0, 0.0, 0.5, 0.0] * 3, np.float32), uniforms(n, 85),
          near=True)


def test_largest_vocabulary():
    n, V = 2, sv.SD_FILTER_MAX_VOCAB
    t, host = values("normal", n, V, "f32", 61)
    check(t.cuda(), host, np.array([0.8, 1.0], np.float32), np.array([0, 3000], np.int32),
          np.array([0.9, 0.99], np.float32), np.zeros(2, np.float32), uniforms(n, 65))


def test_many_rows():
    n, V = 1100, 515
    t, host = values("normal", n, V, "f32", 71)
    check(t.cuda(), host, *options(n, 73), uniforms(n, 75))


def test_in_place_and_same_bits_on_every_run():
    n, V = 6, 40001
    t, _ = values("coarse", n, V, "f32", 81)
    dev = lambda a: torch.from_numpy(a).cuda()
    T, k, p, m = (dev(a) for a in options(n, 83))
    ws = torch.empty(sv.sd_filter_query_size(n, V), dtype=torch.uint8, device="cuda")
    first = None
    for rep in range(4):
        z = t.cuda()
        out = torch.empty_like(z)
        sv.sd_filter_logits(z, out, ws, temperature=T, top_k=k, top_p=p, min_p=m)
        sv.sd_filter_logits(z, z, ws, temperature=T, top_k=k, top_p=p, min_p=m)
        token = torch.empty(n, dtype=torch.int32, device="cuda")
        sv.sd_sample_filtered(t.cuda(), torch.full((n,), 0.37, device="cuda"), token, ws, temperature=T, top_k=k,
                              top_p=p, min_p=m)
        torch.cuda.synchronize()
        assert torch.equal(z, out)
        first = first or (out.clone(), token.clone())
        assert torch.equal(first[0], out) and torch.equal(first[1], token)


def test_filtered_rows_filter_to_themselves_and_draw_alike():
    """softmax of the filtered rows is the distribution drawn from: drawing
    from them without options gives the same tokens for uniforms away from
    the borders (their rounding to fp32 moves those by about 2^-24)."""
    n, V = 64, 9001
    t, _ = values("normal", n, V, "f32", 91)
    z = t.cuda()
    dev = lambda a: torch.from_numpy(a).cuda()
    T, k, p, m = (dev(a) for a in options(n, 93))
    ws = torch.empty(sv.sd_filter_query_size(n, V), dtype=torch.uint8, device="cuda")
    u = torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    rows, kept, kept2 = torch.empty_like(z), torch.empty(n, dtype=torch.int32, device="cuda"), \
        torch.empty(n, dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(kept), torch.empty_like(kept)
    sv.sd_filter_logits(z, rows, ws, temperature=T, top_k=k, top_p=p, min_p=m)
    sv.sd_sample_filtered(z, u, a, ws, temperature=T, top_k=k, top_p=p, min_p=m, kept=kept)
    sv.sd_sample_filtered(rows, u, b, ws, kept=kept2)
    torch.cuda.synchronize()
    assert torch.equal(kept, kept2)
    assert (a != b).sum() <= 1


def test_rows_apart_do_not_touch_each_other():
    """A batch gives each row what the row alone gives, on another stream and
    with a workspace of its own; two such streams at once."""
    n, V = 10, 12345
    t, host = values("normal", n, V, "bf16", 95)
    z = t.cuda()
    T, k, p, m = options(n, 97)
    u = uniforms(n, 99)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    dev = lambda a: torch.from_numpy(a).cuda()
    o = [dev(a) for a in (T, k, p, m, u)]
    ws = [torch.empty(sv.sd_filter_query_size(n, V), dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for rep in range(3):
        for s, w in zip(streams, ws):
            token = torch.empty(n, dtype=torch.int32, device="cuda")
            s.wait_stream(torch.cuda.current_stream())
            sv.sd_sample_filtered(z, o[4], token, w, *o[:4], stream=s)
            outs.append(token)
    torch.cuda.synchronize()
    single = []
    for i in range(n):
        token = torch.empty(1, dtype=torch.int32, device="cuda")
        sv.sd_sample_filtered(z[i:i + 1], o[4][i:i + 1], token, ws[0], *(a[i:i + 1] for a in o[:4]))
        torch.cuda.synchronize()
        single.append(int(token))
    for token in outs:
        assert token.tolist() == single


def test_replayed_graph_follows_its_inputs():
    n, V = 5, 30011
    t, host = values("normal", n, V, "f32", 101)
    z = t.cuda()
    T, k, p, m = options(n, 103)
    o = [torch.from_numpy(a).cuda() for a in (T, k, p, m)]
    u = torch.zeros(n, device="cuda")
    token = torch.empty(n, dtype=torch.int32, device="cuda")
    rows = torch.empty_like(z)
    ws = torch.empty(sv.sd_filter_query_size(n, V), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sv.sd_sample_filtered(z, u, token, ws, *o, stream=s)
        sv.sd_filter_logits(z, rows, ws, *o, stream=s)
    for rep in range(4):
        u.copy_(torch.rand(n, generator=torch.Generator().manual_seed(rep)))
        z.copy_(t * (1.0 + 0.25 * rep))
        o[0].copy_(torch.from_numpy(np.roll(T, rep)))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        token2, rows2 = torch.empty_like(token), torch.empty_like(rows)
        sv.sd_sample_filtered(z, u, token2, ws, *o)
        sv.sd_filter_logits(z, rows2, ws, *o)
        torch.cuda.synchronize()
        assert torch.equal(token, token2) and torch.equal(rows, rows2), rep


def test_refusals_of_tensors():
    z = torch.zeros((2, 8), device="cuda")
    u, token = torch.zeros(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = torch.empty(sv.sd_filter_query_size(2, 8), dtype=torch.uint8, device="cuda")
    for bad in (dict(u=u.double()), dict(u=u[:1]), dict(u=u.cpu()), dict(token=token.long()), dict(logits=z.t()),
                dict(logits=z.half()), dict(logits=z[0]), dict(logits=z[:1].expand(2, 8)), dict(logits=z.cpu())):
        a = dict(logits=z, u=u, token=token)
        a.update(bad)
        with pytest.raises(ValueError):
            sv.sd_sample_filtered(a["logits"], a["u"], a["token"], ws)
    with pytest.raises(ValueError):
        sv.sd_sample_filtered(z, u, token, ws, top_k=torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError):
        sv.sd_filter_logits(z, z[:, :4], ws)
    with pytest.raises(sv.SdError) as e:  # overlaps, but is not in place
        buf = torch.zeros(40, device="cuda")
        sv.sd_filter_logits(buf[:16].view(2, 8), buf[8:24].view(2, 8), ws)
    assert e.value.status == sv.SD_EINVAL
    with pytest.raises(sv.SdError) as e:
        sv.sd_sample_filtered(z, u, token, ws[:0])
    assert e.value.status in (sv.SD_EINVAL, sv.SD_ENOMEM)


def test_rows_beyond_32_bit_offsets():
    n, V, stride = 3, 4099, (1 << 30) + 7
    t, host = values("normal", n, V, "bf16", 111)
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((n, V), (stride, 1))
    z.copy_(t)
    check(z, host, *options(n, 113), uniforms(n, 115))
