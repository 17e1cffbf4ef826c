"""Adapters of many requests beside a shared projection (sd_lora_apply) against
their 64-bit definition (oracle.requests.lora).

Tolerance per output, from the sums' lengths: fp32 sums of d_in and of rank
products are off by at most (d_in + rank + 8) 2^-24 of the sum of absolute
products; in bf16 the inner result is carried on in two bf16 planes, which
keeps it to 2^-17 (twice half a step of the second plane); the output's own rounding
adds half a step of its type.  The 2-norm over all outputs is held to what
roundings of random sign leave of that: square roots of the lengths, times 4."""
import numpy as np
import pytest
import torch

from oracle import requests as rq
from paper_2604_20919_amd import sdverify as sv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(T, d_in, segs, rank, n, dtype="bf16", y_dtype="f32", planes=1, ids=None, seed=0, pad=0):
    r = np.random.default_rng(seed)
    d_out = sum(segs)
    t = lambda *s: torch.from_numpy(r.standard_normal(s).astype(np.float32))
    x = t(T, d_in)
    hi = x.to(DT[dtype])
    c = dict(segs=segs, a=(t(n, len(segs) * rank, d_in) * 0.1).to(DT[dtype]), b=(t(n, d_out, rank) * 0.1).to(DT[dtype]),
             scale=t(n), x=hi, x_lo=(x - hi.float()).to(DT[dtype]) if planes == 2 else None, y=t(T, d_out).to(DT[y_dtype]),
             ids=np.asarray(r.integers(-1, n, T) if ids is None else ids, np.int32))
    return c


def wide(t, pad, offset=0):
    """t on the GPU with rows `pad` further apart and `offset` elements in."""
    if t is None:
        return None
    n, w = t.shape
    buf = torch.full((n * (w + pad) + offset + 1,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf.as_strided((n, w), (w + pad, 1), offset)
    v.copy_(t)
    return v


def apply(c, pad=0, offset=0, in_place=False, stream=None, no_scale=False):
    y = wide(c["y"], pad, offset)
    out = y if in_place else wide(torch.full_like(c["y"], 9.0), pad, offset)
    w = sv.make_lora(c["a"].cuda(), c["b"].cuda(), None if no_scale else c["scale"].cuda(), c["segs"])
    ws = torch.empty(sv.sd_lora_query_size(w, len(c["ids"])), dtype=torch.uint8, device="cuda")
    ids, x, lo = torch.from_numpy(c["ids"]).cuda(), wide(c["x"], pad, offset), wide(c["x_lo"], pad, offset)
    torch.cuda.synchronize()
    sv.sd_lora_apply(w, ids, x, y, out, ws, x_lo=lo, stream=stream)
    torch.cuda.synchronize()
    return out.cpu()


def expect(c, got, no_scale=False):
    x = c["x"].double().numpy() + (0 if c["x_lo"] is None else c["x_lo"].double().numpy())
    a, b = c["a"].double().numpy(), c["b"].double().numpy()
    scale = np.ones(a.shape[0]) if no_scale else c["scale"].double().numpy()
    y = c["y"].double().numpy()
    ref = rq.lora(y, x, c["ids"], a, b, scale, c["segs"])
    size = rq.lora(np.zeros_like(y), np.abs(x), c["ids"], np.abs(a), np.abs(b), np.abs(scale), c["segs"])
    d_in, rank = a.shape[2], b.shape[2]
    bf16 = c["x"].dtype == torch.bfloat16
    eps = torch.finfo(c["y"].dtype).eps / 2
    # (the output is rounded once from an fp32 sum, which for an fp32 output is that rounding)
    tol = size * ((d_in + rank + 8) * 2.0 ** -24 + (2.0 ** -17 if bf16 else 0)) + np.abs(ref) * (eps + 2.0 ** -24)
    err = np.abs(got.double().numpy() - ref)
    assert np.all(err <= tol + 1e-30), (float((err / (tol + 1e-30)).max()), np.unravel_index(np.argmax(err / (tol + 1e-30)), err.shape))
    live = (c["ids"] >= 0) & (c["ids"] < a.shape[0])
    if live.any():
        d = np.linalg.norm((ref - y)[live])
        lim = 4 * d * (np.sqrt(d_in + rank) * 2.0 ** -24 + (2.0 ** -18 if bf16 else 0)) + \
            np.linalg.norm(ref[live]) * (eps + 2.0 ** -24)
        assert np.linalg.norm(err[live]) <= lim, (np.linalg.norm(err[live]), lim)
    assert torch.equal(got[torch.from_numpy(~live)], c["y"][torch.from_numpy(~live)])


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("dtype,y_dtype,planes", [("bf16", "f32", 1), ("bf16", "f32", 2), ("bf16", "bf16", 1), ("f32", "f32", 1)])
def test_row_counts(T, dtype, y_dtype, planes):
    c = make(T, 256, [320], 16, 5, dtype, y_dtype, planes, seed=T)
    expect(c, apply(c))


@pytest.mark.parametrize("rank", [1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 24, 31, 32, 33, 48, 64, 65, 96, 100, 127, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ranks(rank, dtype):
    c = make(37, 200, [176], rank, 3, dtype, seed=rank)
    expect(c, apply(c))
    c = make(21, 136, [64, 16, 48], rank, 3, dtype, seed=rank)
    expect(c, apply(c))


@pytest.mark.parametrize("d_in", [1, 3, 7, 8, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1000, 4099])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_input_widths(d_in, dtype):
    c = make(19, d_in, [96], 8, 4, dtype, planes=2 if dtype == "bf16" else 1, seed=d_in)
    expect(c, apply(c))


@pytest.mark.parametrize("segs", [[1], [2], [7], [15], [16], [17], [63], [65], [129], [1000], [2049], [1, 1], [16, 3, 5],
                                  [100, 1, 30, 7], [256, 64, 64]])
@pytest.mark.parametrize("y_dtype", ["f32", "bf16"])
def test_output_widths_and_segments(segs, y_dtype):
    c = make(23, 72, segs, 8, 4, "bf16", y_dtype, seed=sum(segs))
    expect(c, apply(c))
    c = make(23, 72, segs, 8, 4, "f32", y_dtype, seed=sum(segs))
    expect(c, apply(c))


@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (8, 0), (8, 8), (3, 5), (2, 2), (4, 4), (6, 3)])
@pytest.mark.parametrize("dtype,y_dtype", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
def test_strides_and_alignments(pad, offset, dtype, y_dtype):
    c = make(35, 264, [160, 48], 16, 4, dtype, y_dtype, planes=2 if dtype == "bf16" else 1, seed=pad + offset)
    expect(c, apply(c, pad, offset))
    expect(c, apply(c, pad, offset, in_place=True))


@pytest.mark.parametrize("T,d_in,segs,rank,dtype,y_dtype,planes", [
    (2049, 333, [130, 40, 70], 33, "bf16", "f32", 2), (2500, 640, [200, 64, 64], 64, "bf16", "f32", 2),
    (2177, 1000, [72], 128, "bf16", "bf16", 2), (2300, 129, [100, 30], 65, "bf16", "f32", 1),
    (2048, 1, [1], 1, "bf16", "bf16", 1), (2100, 70, [66, 3], 5, "f32", "bf16", 1), (2200, 257, [140, 64, 64], 43, "f32", "f32", 1),
])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1)])
def test_many_rows(T, d_in, segs, rank, dtype, y_dtype, planes, pad, offset):
    c = make(T, d_in, segs, rank, 4, dtype, y_dtype, planes, seed=T + pad)
    expect(c, apply(c, pad, offset))
    expect(c, apply(c, pad, offset, in_place=True))


@pytest.mark.parametrize("T", [383, 384, 385, 640, 1023])
@pytest.mark.parametrize("n,rank,segs,planes", [(1, 48, [136], 1), (3, 64, [100], 2), (3, 40, [64, 30, 33], 2), (17, 64, [72], 1)])
def test_rows_between_few_and_many(T, n, rank, segs, planes):
    c = make(T, 1160, segs, rank, n, planes=planes, seed=T + n)
    expect(c, apply(c))
    c = make(T, 5000, segs, rank, n, "f32", "bf16", seed=T + n, ids=np.sort(np.random.default_rng(T).integers(-1, n, T)))
    expect(c, apply(c, in_place=True))


@pytest.mark.parametrize("name,ids", [
    ("none", [-1] * 40), ("one", [2] * 40), ("runs", [0] * 17 + [-1] * 3 + [3] * 16 + [1] * 4),
    ("alternating", [0, 1] * 20), ("all apart", list(range(40))), ("out of range", [0, 40, -2, 1 << 30, -(1 << 31), 39] * 6 + [0] * 4),
])
def test_owners_of_rows(name, ids):
    c = make(40, 128, [144], 8, 40, ids=np.asarray(ids, np.int64).astype(np.int32), seed=1)
    expect(c, apply(c))
    expect(c, apply(c, in_place=True, no_scale=True), no_scale=True)


@pytest.mark.parametrize("T,d_in,segs,rank,n,planes,y_dtype", [
    (80, 25600, [5120], 32, 16, 2, "f32"), (229, 5120, [8192, 1024, 1024], 16, 32, 2, "f32"),
    (1, 2048, [2048, 1024, 1024], 16, 4, 1, "f32"), (700, 5120, [5120], 64, 3, 1, "bf16"),
    (2500, 1024, [1040], 64, 3, 2, "f32"), (2048, 520, [600, 40], 20, 2, 1, "bf16"), (4111, 256, [130], 8, 40, 1, "f32"),
])
def test_widths_of_the_models(T, d_in, segs, rank, n, planes, y_dtype):
    r = np.random.default_rng(T)
    c = make(T, d_in, segs, rank, n, "bf16", y_dtype, planes, ids=np.repeat(r.integers(-1, n, T // 3 + 1), 3)[:T], seed=T)
    expect(c, apply(c))


def test_other_rows_and_adapters_do_not_leak():
    """Not-a-numbers in another row, in an adapter that no row has, and in y
    stay where they are."""
    c = make(48, 128, [96], 8, 4, ids=np.arange(48) % 3, seed=9)
    clean = apply(c)
    c["x"][5] = float("nan")
    c["a"][3] = float("nan")
    c["b"][3] = float("inf")
    c["y"][7, 11] = float("nan")
    got = apply(c)
    rows = torch.tensor([t for t in range(48) if t not in (5, 7)])
    assert torch.equal(got[rows], clean[rows])
    assert torch.isnan(got[5]).all() and torch.isnan(got[7, 11])
    at = torch.arange(96) != 11
    assert torch.equal(got[7][at], clean[7][at])
    # a row's values do not depend on its neighbours' adapters either
    c["a"][2] = float("inf")
    c["b"][2] = float("nan")
    got = apply(c)
    rows = torch.tensor([t for t in range(48) if t not in (5, 7) and t % 3 != 2])
    assert torch.equal(got[rows], clean[rows])


@pytest.mark.parametrize("rank,planes,dtype", [(64, 1, "bf16"), (50, 2, "bf16"), (64, 1, "f32")])
def test_many_rows_do_not_leak(rank, planes, dtype):
    T = 1030
    ids = np.arange(T) // 7 % 3
    c = make(T, 136, [96, 40], rank, 4, dtype, planes=planes, ids=ids, seed=rank)
    clean = apply(c)
    c["x"][[5, 700]] = float("nan")
    c["a"][3] = float("nan")
    c["b"][3] = float("inf")
    got = apply(c)
    on = np.ones(T, bool)
    on[[5, 700]] = False
    assert torch.equal(got[torch.from_numpy(on)], clean[torch.from_numpy(on)]) and torch.isnan(got[[5, 700]]).all()
    c["a"][2] = float("inf")
    c["b"][2] = float("nan")
    got = apply(c, in_place=True)
    on &= ids != 2
    assert torch.equal(got[torch.from_numpy(on)], clean[torch.from_numpy(on)])


def test_many_rows_in_a_graph_and_on_two_streams():
    """Replays follow their inputs, with a run of the same sizes beside them."""
    c = make(1300, 512, [256, 128], 40, 3, planes=2, seed=4)
    w = sv.make_lora(c["a"].cuda(), c["b"].cuda(), c["scale"].cuda(), c["segs"])
    ids, x, lo, y = torch.from_numpy(c["ids"]).cuda(), c["x"].cuda(), c["x_lo"].cuda(), c["y"].cuda()
    out, beside = torch.empty_like(y), torch.empty_like(y)
    ws, ws2 = (torch.empty(sv.sd_lora_query_size(w, 1300), dtype=torch.uint8, device="cuda") for _ in range(2))
    s, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sv.sd_lora_apply(w, ids, x, y, out, ws, x_lo=lo, stream=s)
    for rep in range(4):
        ids.copy_(torch.from_numpy(np.roll(c["ids"], 5 * rep)))
        x.copy_(c["x"] * (1 + rep))
        torch.cuda.synchronize()
        g.replay()
        sv.sd_lora_apply(w, ids, x, y, beside, ws2, x_lo=lo, stream=s2)
        torch.cuda.synchronize()
        assert torch.equal(out, beside), rep
        d = dict(c, ids=np.roll(c["ids"], 5 * rep), x=c["x"] * (1 + rep))
        expect(d, out.cpu())


def test_same_bits_alone_and_on_every_run():
    """A run gives the same bits again, in place too, and on another stream
    while one runs beside it."""
    c = make(90, 1024, [512], 16, 6, planes=2, seed=3)
    first = apply(c)
    for s in (None, torch.cuda.Stream()):
        assert torch.equal(first, apply(c, stream=s))
        assert torch.equal(first, apply(c, stream=s, in_place=True))


def test_replayed_graph_follows_its_inputs():
    c = make(30, 512, [256, 128], 16, 5, seed=4)
    w = sv.make_lora(c["a"].cuda(), c["b"].cuda(), c["scale"].cuda(), c["segs"])
    ids, x, y = torch.from_numpy(c["ids"]).cuda(), c["x"].cuda(), c["y"].cuda()
    out = torch.empty_like(y)
    ws, ws2 = (torch.empty(sv.sd_lora_query_size(w, 30), dtype=torch.uint8, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        sv.sd_lora_apply(w, ids, x, y, out, ws, stream=s)
    for rep in range(4):
        ids.copy_(torch.from_numpy(np.roll(c["ids"], rep)))
        x.copy_(c["x"] * (1 + rep))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        ref = torch.empty_like(y)
        sv.sd_lora_apply(w, ids, x, y, ref, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, ref), rep


def test_refusals_of_tensors():
    c = make(6, 64, [48], 8, 3, seed=5)
    a, b, sc = c["a"].cuda(), c["b"].cuda(), c["scale"].cuda()
    for bad in (dict(b=b.float()), dict(segs=[40]), dict(segs=[24, 24]), dict(a=a[0]), dict(scale=sc[:2]), dict(a=a.cpu()),
                dict(b=b.transpose(1, 2)), dict(a=a[:, ::2])):
        k = dict(a=a, b=b, scale=sc, segs=None)
        k.update(bad)
        with pytest.raises(ValueError):
            sv.make_lora(**k)
    w = sv.make_lora(a, b, sc)
    x, y, ids = c["x"].cuda(), c["y"].cuda(), torch.from_numpy(c["ids"]).cuda()
    ws = torch.empty(sv.sd_lora_query_size(w, 6), dtype=torch.uint8, device="cuda")
    for bad in (dict(x=x.float()), dict(x=x[:, :32]), dict(y_out=y.bfloat16()), dict(adapter=ids.long()), dict(adapter=ids[:3]),
                dict(y_in=y[:3]), dict(x_lo=x[:3]), dict(y_out=y[:1].expand(6, 48)), dict(x=x.cpu())):
        k = dict(adapter=ids, x=x, y_in=y, y_out=torch.empty_like(y), workspace=ws)
        k.update(bad)
        with pytest.raises(ValueError):
            sv.sd_lora_apply(w, **k)
    with pytest.raises(sv.SdError) as e:  # overlaps, but is not in place
        buf = torch.zeros(6 * 48 + 48, device="cuda")
        sv.sd_lora_apply(w, ids, x, buf[:288].view(6, 48), buf[48:].view(6, 48), ws)
    assert e.value.status == sv.SD_EINVAL


def test_rows_beyond_32_bit_offsets():
    c = make(3, 72, [40], 8, 2, ids=[1, -1, 0], seed=6)
    stride = (1 << 30) + 9
    far = lambda t: torch.empty(2 * stride + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (stride, 1))
    w = sv.make_lora(c["a"].cuda(), c["b"].cuda(), c["scale"].cuda(), c["segs"])
    x, y = far(c["x"]), far(c["y"].bfloat16())
    c["y"] = c["y"].bfloat16()
    x.copy_(c["x"])
    y.copy_(c["y"])
    ws = torch.empty(sv.sd_lora_query_size(w, 3), dtype=torch.uint8, device="cuda")
    sv.sd_lora_apply(w, torch.from_numpy(c["ids"]).cuda(), x, y, y, ws)
    torch.cuda.synchronize()
    expect(c, y.cpu())


@pytest.mark.parametrize("T,n", [(1 << 20, 1), (1 << 20, 40), (8191, 40)])
def test_most_rows(T, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(T + n)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    a, b, scale, x, y = r(n, 2, 8), r(n, 8, 2), r(n), r(T, 8), r(T, 8)
    ids = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    w = sv.make_lora(a, b, scale)
    out = torch.empty_like(y)
    ws = torch.empty(sv.sd_lora_query_size(w, T), dtype=torch.uint8, device="cuda")
    sv.sd_lora_apply(w, ids, x, y, out, ws)
    on, i = (ids >= 0)[:, None], ids.clamp(min=0).long()
    d = lambda t: t.double()
    f = lambda a, x, b, s: (b[i] * (a[i] * x[:, None, :]).sum(2)[:, None, :]).sum(2) * s[i][:, None]
    ref = torch.where(on, d(y) + f(d(a), d(x), d(b), d(scale)), d(y))
    size = torch.where(on, f(d(a).abs(), d(x).abs(), d(b).abs(), d(scale).abs()), 0.0)
    # (as in expect: an fp32 sum of 8 and 2 products and its rounding)
    tol = size * (8 + 2 + 8) * 2.0 ** -24 + ref.abs() * 2.0 ** -23
    assert bool(((d(out) - ref).abs() <= tol).all())
