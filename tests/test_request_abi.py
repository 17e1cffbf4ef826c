"""Refusals of the calls for a request's own sampling options and adapters, all
made on the host before anything is enqueued.  No call here touches a GPU."""
import ctypes

import pytest

from paper_2604_20919_amd import sdverify as sv

P = ctypes.c_void_p(4096)  # never dereferenced: every call below is refused first


def _size(n, v):
    b = ctypes.c_uint64()
    return sv.lib().sd_filter_query_size(n, v, ctypes.byref(b)), b.value


def test_filter_sizes():
    assert _size(0, 5)[0] == sv.SD_EINVAL and _size(5, 0)[0] == sv.SD_EINVAL and _size(-1, 5)[0] == sv.SD_EINVAL
    assert _size(sv.SD_FILTER_MAX_ROWS + 1, 5)[0] == sv.SD_ELIMIT
    assert _size(1, sv.SD_FILTER_MAX_VOCAB + 1)[0] == sv.SD_ELIMIT
    assert sv.lib().sd_filter_query_size(1, 1, None) == sv.SD_EINVAL
    for n, v in ((1, 1), (sv.SD_FILTER_MAX_ROWS, sv.SD_FILTER_MAX_VOCAB), (416, 151936)):
        s, b = _size(n, v)
        assert s == sv.SD_OK and b > 0
    assert sv.sd_filter_query_size(3, 1000) > 0


@pytest.mark.parametrize("bad,status", [
    (dict(n=0), sv.SD_EINVAL), (dict(v=0), sv.SD_EINVAL), (dict(z=None), sv.SD_EINVAL), (dict(dt=2), sv.SD_EINVAL),
    (dict(stride=99), sv.SD_EINVAL), (dict(u=None), sv.SD_EINVAL), (dict(token=None), sv.SD_EINVAL),
    (dict(ws=None), sv.SD_EINVAL), (dict(ws=ctypes.c_void_p(4098)), sv.SD_EINVAL), (dict(size=0), sv.SD_ENOMEM),
    (dict(z=ctypes.c_void_p(4097)), sv.SD_EINVAL), (dict(u=ctypes.c_void_p(4098)), sv.SD_EINVAL),
    (dict(n=sv.SD_FILTER_MAX_ROWS + 1), sv.SD_ELIMIT), (dict(prob=ctypes.c_void_p(4097)), sv.SD_EINVAL),
])
def test_sample_refusals(bad, status):
    k = dict(n=2, v=100, z=P, dt=0, stride=100, u=P, token=P, prob=None, ws=P, size=1 << 40)
    k.update(bad)
    f = sv.sd_filter()
    assert sv.lib().sd_sample_filtered(k["n"], k["v"], k["z"], k["dt"], k["stride"], ctypes.byref(f), k["u"], k["token"],
                                       k["prob"], None, k["ws"], k["size"], None) == status


@pytest.mark.parametrize("bad", [dict(out=None), dict(ostride=99), dict(out=ctypes.c_void_p((1 << 20) + 4)),
                                 dict(out=ctypes.c_void_p((1 << 20) + 2)), dict(dt=1, out=ctypes.c_void_p(1 << 20)),
                                 dict(ostride=104), dict(opt=ctypes.c_void_p(4097))])
def test_filter_logits_refusals(bad):
    z = ctypes.c_void_p(1 << 20)
    k = dict(out=z, ostride=100, dt=0, opt=None)
    k.update(bad)
    f = sv.sd_filter(None, k["opt"], None, None)
    assert sv.lib().sd_filter_logits(2, 100, z, k["dt"], 100, ctypes.byref(f), k["out"], k["ostride"], None, P, 1 << 40,
                                     None) == sv.SD_EINVAL


def _lora(**kw):
    k = dict(n=3, rank=8, d_in=64, d_out=48, segs=[0, 48], dtype=sv.SD_BF16, a=P, b=P, n_seg=None)
    k.update(kw)
    off = (ctypes.c_int32 * (sv.SD_LORA_MAX_SEGS + 1))(*k["segs"][:sv.SD_LORA_MAX_SEGS + 1])
    return sv.sd_lora(k["n"], k["rank"], k["d_in"], k["d_out"], k["n_seg"] or len(k["segs"]) - 1, off, k["dtype"], k["a"],
                      k["b"], None)


@pytest.mark.parametrize("bad,status", [
    (dict(n=0), sv.SD_EINVAL), (dict(rank=0), sv.SD_EINVAL), (dict(d_in=0), sv.SD_EINVAL), (dict(d_out=0), sv.SD_EINVAL),
    (dict(dtype=2), sv.SD_EINVAL), (dict(segs=[0, 47]), sv.SD_EINVAL), (dict(segs=[1, 48]), sv.SD_EINVAL),
    (dict(segs=[0, 48, 48]), sv.SD_EINVAL), (dict(segs=[0, 30, 20, 48]), sv.SD_EINVAL),
    (dict(rank=sv.SD_LORA_MAX_RANK + 1), sv.SD_ELIMIT), (dict(n_seg=sv.SD_LORA_MAX_SEGS + 1), sv.SD_ELIMIT),
    (dict(d_in=(1 << 20) + 1), sv.SD_ELIMIT), (dict(d_out=(1 << 20) + 1, segs=[0, (1 << 20) + 1]), sv.SD_ELIMIT),
])
def test_lora_descriptor_refusals(bad, status):
    b = ctypes.c_uint64()
    w = _lora(**bad)
    assert sv.lib().sd_lora_query_size(ctypes.byref(w), 4, ctypes.byref(b)) == status
    assert sv.lib().sd_lora_apply(ctypes.byref(w), 4, P, P, None, 1 << 21, P, 1 << 21, P, 1 << 21, 0, P, 1 << 40,
                                  None) == status


def test_lora_sizes():
    b = ctypes.c_uint64()
    w = _lora()
    assert sv.lib().sd_lora_query_size(None, 4, ctypes.byref(b)) == sv.SD_EINVAL
    assert sv.lib().sd_lora_query_size(ctypes.byref(w), 0, ctypes.byref(b)) == sv.SD_EINVAL
    assert sv.lib().sd_lora_query_size(ctypes.byref(w), (1 << 20) + 1, ctypes.byref(b)) == sv.SD_ELIMIT
    assert sv.lib().sd_lora_query_size(ctypes.byref(w), 1 << 20, ctypes.byref(b)) == sv.SD_OK and b.value > 0


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), sv.SD_EINVAL), (dict(ids=None), sv.SD_EINVAL), (dict(yi=None), sv.SD_EINVAL), (dict(yo=None), sv.SD_EINVAL),
    (dict(xs=63), sv.SD_EINVAL), (dict(ys=47), sv.SD_EINVAL), (dict(yos=47), sv.SD_EINVAL), (dict(yd=2), sv.SD_EINVAL),
    (dict(x=ctypes.c_void_p(4097)), sv.SD_EINVAL), (dict(yo=ctypes.c_void_p((1 << 20) + 2)), sv.SD_EINVAL),
    (dict(yo=ctypes.c_void_p((1 << 20) + 4)), sv.SD_EINVAL), (dict(yos=49), sv.SD_EINVAL), (dict(ws=None), sv.SD_EINVAL),
    (dict(ws=ctypes.c_void_p(4352 + 128)), sv.SD_EINVAL), (dict(size=16), sv.SD_ENOMEM),
])
def test_lora_refusals(bad, status):
    y = ctypes.c_void_p(1 << 20)
    k = dict(ids=P, x=P, lo=None, xs=64, yi=y, ys=48, yo=y, yos=48, yd=0, ws=P, size=1 << 40)
    k.update(bad)
    w = _lora()
    assert sv.lib().sd_lora_apply(ctypes.byref(w), 4, k["ids"], k["x"], k["lo"], k["xs"], k["yi"], k["ys"], k["yo"],
                                  k["yos"], k["yd"], k["ws"], k["size"], None) == status


def test_lora_second_plane_is_for_bf16():
    w = _lora(dtype=sv.SD_F32)
    y = ctypes.c_void_p(1 << 20)
    assert sv.lib().sd_lora_apply(ctypes.byref(w), 4, P, P, P, 64, y, 48, y, 48, 0, P, 1 << 40, None) == sv.SD_EINVAL
