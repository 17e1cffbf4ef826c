"""Refusals of the calls for trees of drafts, cache pages and rules on logits, all
made on the host before anything is enqueued.  No call here touches a GPU."""
import ctypes

import pytest

from paper_2604_20919_amd import sdverify as sv

P = ctypes.c_void_p(4096)  # never dereferenced: every call below is refused first
BIG = 1 << 62


def pool(**kw):
    k = dict(layers=2, pages=64, heads=4, hd=128, dtype=sv.SD_BF16, base=4096)
    k.update(kw)
    return sv.sd_kv_pool(k["layers"], k["pages"], k["heads"], k["hd"], k["dtype"], k["base"])


def tree(**kw):
    k = dict(users=3, slots=12, max_slots=8, max_pages=10, off=4096, prefix=4096, table=4096, parent=4096)
    k.update(kw)
    return sv.sd_tree(k["users"], k["slots"], k["max_slots"], k["max_pages"], k["off"], k["prefix"], k["table"], k["parent"])


POOLS = [(dict(layers=0), sv.SD_EINVAL), (dict(pages=0), sv.SD_EINVAL), (dict(heads=0), sv.SD_EINVAL),
         (dict(hd=0), sv.SD_EINVAL), (dict(dtype=2), sv.SD_EINVAL), (dict(hd=96), sv.SD_ENOTIMPL),
         (dict(hd=256), sv.SD_ENOTIMPL), (dict(hd=33, dtype=sv.SD_F32), sv.SD_ENOTIMPL),
         (dict(hd=130, dtype=sv.SD_F32), sv.SD_ENOTIMPL), (dict(pages=(1 << 27) + 1), sv.SD_ELIMIT),
         (dict(heads=(1 << 13) + 1), sv.SD_ELIMIT), (dict(layers=(1 << 12) + 1), sv.SD_ELIMIT)]
TREES = [(dict(users=0), sv.SD_EINVAL), (dict(slots=0), sv.SD_EINVAL), (dict(max_slots=0), sv.SD_EINVAL),
         (dict(max_pages=0), sv.SD_EINVAL), (dict(max_slots=sv.SD_TREE_MAX_SLOTS + 1), sv.SD_ELIMIT),
         (dict(users=sv.SD_TREE_MAX_USERS + 1), sv.SD_ELIMIT), (dict(slots=(1 << 20) + 1), sv.SD_ELIMIT)]


def attention(po, tr, **kw):
    k = dict(layer=1, hq=8, q=1 << 24, q_lo=None, qs=1024, out=1 << 25, out_lo=None, os=1024, scale=0.1, ws=1 << 26, size=BIG)
    k.update(kw)
    return sv.lib().sd_tree_attention(ctypes.byref(po), k["layer"], ctypes.byref(tr), k["hq"], k["q"], k["q_lo"], k["qs"],
                                      k["out"], k["out_lo"], k["os"], k["scale"], k["ws"], k["size"], None)


@pytest.mark.parametrize("bad,status", POOLS)
def test_pool_refusals(bad, status):
    po, b = pool(**bad), ctypes.c_uint64()
    assert sv.lib().sd_tree_query_size(ctypes.byref(po), ctypes.byref(tree()), 8, ctypes.byref(b)) == status
    assert attention(po, tree()) == status
    assert sv.lib().sd_kv_copy_pages(ctypes.byref(po), 1, P, P, None) == status
    assert sv.lib().sd_kv_compact(ctypes.byref(po), 1, P, P, 1, P, 1, P, None) == status


@pytest.mark.parametrize("bad,status", TREES)
def test_tree_refusals(bad, status):
    tr, b = tree(**bad), ctypes.c_uint64()
    assert sv.lib().sd_tree_query_size(ctypes.byref(pool()), ctypes.byref(tr), 8, ctypes.byref(b)) == status
    assert attention(pool(), tr) == status


def test_tree_sizes():
    b = ctypes.c_uint64()
    q = lambda hq, t=tree(), p=pool(): (sv.lib().sd_tree_query_size(ctypes.byref(p), ctypes.byref(t), hq, ctypes.byref(b)), b.value)  # noqa: E731,B008
    assert q(7)[0] == sv.SD_EINVAL and q(0)[0] == sv.SD_EINVAL and q(4 * 129)[0] == sv.SD_ELIMIT
    assert sv.lib().sd_tree_query_size(ctypes.byref(pool()), ctypes.byref(tree()), 8, None) == sv.SD_EINVAL
    assert sv.lib().sd_tree_query_size(None, ctypes.byref(tree()), 8, ctypes.byref(b)) == sv.SD_EINVAL
    assert sv.lib().sd_tree_query_size(ctypes.byref(pool()), None, 8, ctypes.byref(b)) == sv.SD_EINVAL
    assert q(8)[0] == sv.SD_OK and q(8)[1] > 0
    # the widest launch the limits admit
    s, most = q(128 << 13, tree(users=sv.SD_TREE_MAX_USERS, slots=1 << 20, max_slots=256, max_pages=1 << 27),
                pool(pages=1 << 27, heads=1 << 13))
    assert s in (sv.SD_OK, sv.SD_ELIMIT)


@pytest.mark.parametrize("bad", [
    dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(ws=None), dict(qs=1023), dict(os=1016), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=(1 << 24) + 8), dict(out=(1 << 25) + 2),
    dict(q_lo=(1 << 23) + 4), dict(out_lo=(1 << 23) + 4), dict(qs=1028), dict(os=1025), dict(ws=(1 << 26) + 128),
    dict(out=1 << 24), dict(out=(1 << 24) + 11 * 2048), dict(out_lo=1 << 25), dict(out_lo=1 << 24), dict(q_lo=1 << 25),
    dict(hq=6),
])
def test_attention_refusals(bad):
    assert attention(pool(), tree(), **bad) == sv.SD_EINVAL


def test_attention_refusals_of_arrays_and_workspace():
    for name in ("off", "prefix", "table"):
        assert attention(pool(), tree(**{name: None})) == sv.SD_EINVAL
        assert attention(pool(), tree(**{name: 4098})) == sv.SD_EINVAL
    assert attention(pool(), tree(parent=4097)) == sv.SD_EINVAL
    assert attention(pool(base=None), tree()) == sv.SD_EINVAL
    assert attention(pool(base=4096 + 128), tree()) == sv.SD_EINVAL
    assert attention(pool(), tree(), size=0) == sv.SD_ENOMEM
    # second planes belong to bf16
    f32 = pool(dtype=sv.SD_F32)
    assert attention(f32, tree(), q_lo=1 << 23) == sv.SD_EINVAL
    assert attention(f32, tree(), out_lo=1 << 23) == sv.SD_EINVAL


def test_page_refusals():
    po = pool()
    call = lambda n=2, s=P, d=P, p=po: sv.lib().sd_kv_copy_pages(ctypes.byref(p), n, s, d, None)  # noqa: E731
    odd = ctypes.c_void_p(4098)
    assert call(n=0) == sv.SD_EINVAL and call(s=None) == sv.SD_EINVAL and call(d=None) == sv.SD_EINVAL
    assert call(s=odd) == sv.SD_EINVAL and call(d=odd) == sv.SD_EINVAL
    assert call(p=pool(base=None)) == sv.SD_EINVAL and call(p=pool(base=64)) == sv.SD_EINVAL
    assert call(n=1 << 21) == sv.SD_ELIMIT  # pages of 32 KB
    assert sv.lib().sd_kv_copy_pages(None, 1, P, P, None) == sv.SD_EINVAL


@pytest.mark.parametrize("bad,status", [
    (dict(n=0), sv.SD_EINVAL), (dict(prefix=None), sv.SD_EINVAL), (dict(table=None), sv.SD_EINVAL), (dict(pages=0), sv.SD_EINVAL),
    (dict(keep=None), sv.SD_EINVAL), (dict(most=0), sv.SD_EINVAL), (dict(n_keep=None), sv.SD_EINVAL),
    (dict(keep=ctypes.c_void_p(4097)), sv.SD_EINVAL), (dict(n_keep=ctypes.c_void_p(4097)), sv.SD_EINVAL),
    (dict(prefix=ctypes.c_void_p(4097)), sv.SD_EINVAL), (dict(table=ctypes.c_void_p(4097)), sv.SD_EINVAL),
    (dict(most=sv.SD_KV_COMPACT_MAX + 1), sv.SD_ELIMIT), (dict(n=sv.SD_TREE_MAX_USERS + 1), sv.SD_ELIMIT),
])
def test_compact_refusals(bad, status):
    k = dict(n=2, prefix=P, table=P, pages=4, keep=P, most=4, n_keep=P)
    k.update(bad)
    assert sv.lib().sd_kv_compact(ctypes.byref(pool()), k["n"], k["prefix"], k["table"], k["pages"], k["keep"], k["most"],
                                  k["n_keep"], None) == status


def rules(**kw):
    r = sv.sd_logit_rules()
    for k, v in kw.items():
        setattr(r, k, v)
    return r


@pytest.mark.parametrize("bad,status", [
    (dict(tokens=4096, n_tokens=4), sv.SD_EINVAL), (dict(hist=4096, n_tokens=4), sv.SD_EINVAL),
    (dict(row_token=4096), sv.SD_EINVAL), (dict(row_parent=4096), sv.SD_EINVAL), (dict(bias=4096, n_bias=1), sv.SD_EINVAL),
    (dict(bias=4096, n_bias=1, bias_token=4096), sv.SD_EINVAL), (dict(bias_token=4096, bias_value=4096, n_bias=1), sv.SD_EINVAL),
    (dict(mask=4096, n_masks=1), sv.SD_EINVAL), (dict(mask_row=4096, n_masks=1), sv.SD_EINVAL),
    (dict(n_tokens=-1), sv.SD_EINVAL), (dict(n_bias=-1), sv.SD_EINVAL), (dict(n_masks=-1), sv.SD_EINVAL),
    (dict(repetition=4097), sv.SD_EINVAL), (dict(presence=4097), sv.SD_EINVAL), (dict(frequency=4098), sv.SD_EINVAL),
    (dict(tokens=4097, hist=4096, n_tokens=4), sv.SD_EINVAL), (dict(tokens=4096, hist=4096, n_tokens=1 << 31), sv.SD_ELIMIT),
    (dict(tokens=4096, hist=4096, n_tokens=(1 << 30) - 4095), sv.SD_ELIMIT),
    (dict(bias=4096, bias_token=4096, bias_value=4096, n_bias=(1 << 30) - 4095), sv.SD_ELIMIT),
    (dict(bias=4096, bias_token=4096, bias_value=4096, n_bias=1 << 31), sv.SD_ELIMIT),
])
def test_rules_refusals(bad, status):
    z = ctypes.c_void_p(1 << 20)
    r = rules(**bad)
    assert sv.lib().sd_adjust_logits(2, 100, z, 0, 100, ctypes.byref(r), z, 100, None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(n=0), sv.SD_EINVAL), (dict(v=0), sv.SD_EINVAL), (dict(z=None), sv.SD_EINVAL), (dict(out=None), sv.SD_EINVAL),
    (dict(dt=2), sv.SD_EINVAL), (dict(stride=99), sv.SD_EINVAL), (dict(ostride=99), sv.SD_EINVAL), (dict(r=None), sv.SD_EINVAL),
    (dict(z=(1 << 20) + 2), sv.SD_EINVAL), (dict(out=(1 << 20) + 2), sv.SD_EINVAL), (dict(out=(1 << 20) + 4), sv.SD_EINVAL),
    (dict(ostride=104), sv.SD_EINVAL), (dict(dt=1), sv.SD_EINVAL), (dict(n=sv.SD_FILTER_MAX_ROWS + 1), sv.SD_ELIMIT),
    (dict(v=sv.SD_FILTER_MAX_VOCAB + 1, stride=1 << 21, ostride=1 << 21), sv.SD_ELIMIT),
])
def test_adjust_refusals(bad, status):
    k = dict(n=2, v=100, z=1 << 20, dt=0, stride=100, out=1 << 20, ostride=100, r=rules())
    k.update(bad)
    r = None if k["r"] is None else ctypes.byref(k["r"])
    assert sv.lib().sd_adjust_logits(k["n"], k["v"], k["z"], k["dt"], k["stride"], r, k["out"], k["ostride"], None) == status
