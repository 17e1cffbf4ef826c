"""Sampling options and adapters in contexts whose own buffers are small: the
filter takes a batch a few rows at a time, the adapters' inner results outgrow
the logits, and neither disturbs the pass."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
import workload as wl
from gpu_harness import assert_decisions, compare_decisions, logit_rel_err
from paper_2604_20919_amd import sdverify as sv
from test_gpu_requests import OPTIONS, Adapters, context, filtered, reference, verify
from test_gpu_sampler import _case, _sampler_verifier

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,base,over", [
    ("small-fp32", "tiny", dict(vocab=40002, d_ffn=256)),           # a few rows at a time
    ("small-vocab", "tiny-bf16", dict(vocab=512, d_model=2048)),    # inner results beyond the logits
    ("one-chunk", "tiny", dict(vocab=5, d_model=64, n_q_heads=2, n_kv_heads=1, head_dim=32, d_ffn=64)),
])
def test_options_and_adapters_in_small_contexts(name, base, over, monkeypatch):
    monkeypatch.setitem(wl.MODELS, name, dataclasses.replace(wl.MODELS[base], name=name, **over))
    prefix, L = [40, 30, 0, 17, 5, 9, 3, 21], [1, 7, 3, 5, 2, 4, 6, 7]
    w, dw, v = context(name, prefix, L, seed=127)
    b = w.batch(0)
    raw, acc0, tok0 = verify(v, w, b)
    opts = [OPTIONS[i % 6] for i in range(8)]
    for u, o in zip(b.users, opts):
        v.user_sampling(int(u), *o)
    for rep in range(3):
        lg, acc, tok = verify(v, w, b, seed=rep)
        assert np.array_equal(lg, filtered(raw, opts, b.n_slots))
        ref = oracle.sample("stochastic", b.users, b.draft_len, lg, b.drafts, b.q, b.accept_u, rep, 0)
        assert_decisions(compare_decisions(acc, tok, ref, b.draft_len, drafts=b.drafts), f"{name} {rep}", end_to_end=False)
    for u in b.users:
        v.user_sampling(int(u))
    ad = Adapters(w.model, 2, 128 if name == "small-vocab" else 8, seed=3, sigma=0.02)
    v.set_adapters(ad.layers)
    ids = [i % 3 - 1 for i in range(8)]
    for u, a in zip(b.users, ids):
        v.user_adapter(int(u), a)
    got, _, _ = verify(v, w, b)
    err = logit_rel_err(got, reference(w, b, ad, ids))
    assert err.max() < (1e-4 if w.model.dtype == "f32" else 2.3e-3), err.max()
    mine = np.repeat(np.asarray(ids) >= 0, b.n_slots)
    assert np.array_equal(got[~mine], raw[~mine])
    v.set_adapters(None)
    back, acc1, tok1 = verify(v, w, b)
    assert np.array_equal(back, raw) and np.array_equal(acc0, acc1) and np.array_equal(tok0, tok1)
    v.close()


def test_rows_at_a_time_give_the_same_tokens():
    """151936 tokens in a context with small buffers, 29 rows in several goes."""
    Ls = [1, 4, 2, 8, 3, 5]
    logits, q, drafts, au, users = _case(151936, Ls, "stochastic", 83, True)
    v = _sampler_verifier(151936, 6, 8, 29)
    assert v.ws_bytes < 2 * (logits.nbytes + 29 * sv.sd_filter_query_size(1, 151936))  # (two pending batches)
    for u, o in zip(users, OPTIONS):
        v.user_sampling(int(u), *o)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    v.sample(0, np.zeros(6, np.int32), Ls, dev(drafts), dev(q), dev(logits), "stochastic", seed=5, round_=1, accept_u=dev(au))
    acc, tok = v.accept(0, 6)
    ref = oracle.sample("stochastic", users, Ls, filtered(logits, OPTIONS, np.asarray(Ls) + 1), drafts, q, au, 5, 1)
    assert_decisions(compare_decisions(acc, tok, ref, Ls, drafts=drafts), "few rows at a time", end_to_end=False)
    v.close()
