"""The adapters that a context reads in place stay what they were when the
caller's list changes, until they are replaced."""
import gc
import weakref

import numpy as np
import pytest
import torch

from paper_2604_20919_amd import sdverify as sv
from test_gpu_requests import Adapters, context, verify

pytestmark = pytest.mark.gpu


def test_adapters_outlive_the_callers_list():
    w, dw, v = context("tiny-bf16", [30, 4], [4, 2], seed=121)
    b = w.batch(0)
    ad = Adapters(w.model, 2, 8, seed=7)
    layers = ad.layers
    sv.sd_adapters_set(v.ctx, layers)
    for u in range(2):
        v.user_adapter(u, u)
    first, _, _ = verify(v, w, b)
    held = [weakref.ref(x) for l in layers for x in (l["qkv"].a, l["qkv"].b, l["qkv"].scale, l["down"].a)]
    for l in layers:
        l.clear()
    del layers[:]
    gc.collect()
    junk = [torch.full((1 << 16,), 7.0, device="cuda") for _ in range(32)]
    again, _, _ = verify(v, w, b)
    assert np.array_equal(first, again) and all(r() is not None for r in held)
    with pytest.raises(ValueError):
        sv.sd_adapters_set(v.ctx, [{}])  # refused: the set stays
    again, _, _ = verify(v, w, b)
    assert np.array_equal(first, again)
    v.set_adapters(None)
    gc.collect()
    assert all(r() is None for r in held)
    del junk
    v.close()
    assert v.ctx is None
