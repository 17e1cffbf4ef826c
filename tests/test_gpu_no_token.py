"""Users whose rows leave no token to draw -- logits of -inf or not-a-numbers
alone, as a filter or a broken product leaves them.  They get token -1, as in
sd_sample_filtered, and stay where they are on a commit; the other users of
their batch get what they get without them."""
import numpy as np
import pytest
import torch

import workload as wl
from gpu_harness import make_verifier
from paper_2604_20919_amd import sdverify as sv
from paper_2604_20919_amd.draft_loop import DraftLoop
from paper_2604_20919_amd.serve import GpuVerify
from test_gpu_requests import Adapters, context
from test_gpu_sampler import _case, _sampler_verifier

pytestmark = pytest.mark.gpu

LS = [1, 4, 2, 3]
dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731


def rows(V, bad, slot):
    """A case of four users; slot `slot` of users 1 and 3 holds nothing but `bad`."""
    logits, q, drafts, au, users = _case(V, LS, "stochastic", 5, True)
    off = np.cumsum([0] + [l + 1 for l in LS])
    doff = np.cumsum([0] + LS)
    spoilt = logits.copy()
    for u in (1, 3):
        spoilt[off[u] + slot] = bad
    return logits, spoilt, q, drafts, au, doff


@pytest.mark.parametrize("options", [False, True])
@pytest.mark.parametrize("bad", [-np.inf, np.nan])
@pytest.mark.parametrize("slot", [0, 2])
def test_rows_without_a_token(bad, slot, options):
    V = 1024
    logits, spoilt, q, drafts, au, doff = rows(V, bad, slot)
    au = au.copy()
    for u in (1, 3):  # every draft before the spoilt row is accepted
        au[doff[u]:doff[u + 1]] = -1.0
    v = _sampler_verifier(V, 4, 8, sum(LS) + 4)
    if options:
        for u in range(4):
            v.user_sampling(u, 0.8, 40, 0.95, 0.0)
    got = []
    for z in (logits, spoilt):
        v.sample(0, np.zeros(4, np.int32), LS, dev(drafts), dev(q), dev(z), "stochastic", seed=5, round_=1, accept_u=dev(au))
        got.append(v.accept(0, 4))
    (acc0, tok0), (acc, tok) = got
    assert np.all(tok0 >= 0)
    for u in (0, 2):
        assert acc[u] == acc0[u] and tok[u] == tok0[u]
    for u in (1, 3):
        assert acc[u] == slot and tok[u] == -1
    v.close()
    # the filtered draw says the same of such a row
    ws = torch.empty(sv.sd_filter_query_size(1, V), dtype=torch.uint8, device="cuda")
    t = torch.zeros(1, dtype=torch.int32, device="cuda")
    sv.sd_sample_filtered(torch.full((1, V), float(bad), device="cuda"), torch.zeros(1, device="cuda"), t, ws)
    assert int(t) == -1


@pytest.mark.parametrize("bad", [-np.inf, np.nan])
def test_rows_without_a_token_in_the_context_free_sampler(bad):
    V = 4099
    logits, spoilt, q, drafts, au, _ = rows(V, bad, 0)
    out = torch.zeros(9, dtype=torch.int32, device="cuda")
    got = []
    for z in (logits, spoilt):
        sv.sd_sample_logits_noalloc([3, 5, 8, 9], LS, V, dev(drafts), dev(q), dev(z), "stochastic", out, seed=2)
        got.append(out.cpu().numpy())
    assert got[1][8] == 0 and list(got[1][[1, 3, 5, 7]]) == [0, 0, -1, -1]
    assert np.array_equal(got[0][[0, 2, 4, 6]], got[1][[0, 2, 4, 6]])


def spoiled(v, m):
    """Adapter 1 beside the last layer's down projection makes a user's logits
    not-a-numbers (its cached keys and values stay finite)."""
    ad = Adapters(m, 2, 4, seed=3, targets=("down",))
    ad.layers[0] = {}
    ad.layers[-1]["down"].scale[1] = float("nan")
    v.set_adapters(ad.layers)


@pytest.mark.parametrize("options", [False, True])
def test_users_without_a_token_stay_where_they_are(options):
    prefix, L = [12, 40, 7], [2, 3, 1]
    w, dw, v = context("tiny-bf16", prefix, L, seed=101)
    b = w.batch(0)
    drafts, q = dev(b.drafts), dev(b.q)
    V = w.model.vocab
    spoiled(v, w.model)

    def reset():
        for i, u in enumerate(b.users):
            v.reset_user(int(u), int(b.prefix_len[i]), int(b.root[i]))

    if options:
        for u in range(3):
            v.user_sampling(u, 0.7, 0, 0.9, 0.0)
    reset()
    v.verify(0, w.assign, w.draft_len, drafts, q, "stochastic", seed=4)
    acc0, tok0 = v.accept(0, 3)
    v.user_adapter(1, 1)
    probs = torch.full((3, V), 7.0, device="cuda")
    v.draft(0, w.assign, "stochastic", seed=1, probs=probs)
    dacc, dtok = v.accept(0, 3, commit=True)
    assert dtok[1] == -1 and dtok[0] >= 0 and dtok[2] >= 0
    assert v.user_state(1) == (int(b.prefix_len[1]), int(b.root[1]))
    assert v.user_state(0) == (int(b.prefix_len[0]) + 1, int(dtok[0]))
    p = probs.cpu().numpy()
    assert np.all(np.abs(p[[0, 2]].sum(1) - 1) < 1e-4)
    assert np.all(p[1] == 0)
    reset()
    v.verify(0, w.assign, w.draft_len, drafts, q, "stochastic", seed=4)
    acc, tok = v.accept(0, 3, commit=True)
    assert acc[1] == 0 and tok[1] == -1
    assert v.user_state(1) == (int(b.prefix_len[1]), int(b.root[1]))
    for u in (0, 2):
        assert (acc[u], tok[u]) == (acc0[u], tok0[u])
        assert v.user_state(u) == (int(b.prefix_len[u]) + 1 + acc[u], int(tok[u]))
    # and it goes on once it is mended
    v.user_adapter(1, 0)
    v.verify(0, [-1, 0, -1], [1, 3, 1], drafts[2:5], q[2:5].contiguous(), "stochastic", seed=4)
    acc, tok = v.accept(0, 3, commit=True)
    assert tok[1] >= 0 and v.user_state(1) == (int(b.prefix_len[1]) + 1 + acc[1], int(tok[1]))
    v.close()


def test_drafting_loop_with_a_user_without_a_token():
    prefix, L = [33, 7, 90], [3, 2, 4]
    w, dw, dv = context("tiny-bf16", prefix, L, seed=103, max_batch_tokens=15)
    tv = make_verifier(w, dw, extra_ctx=32, max_batch_tokens=15)
    for u in range(3):
        tv.reset_user(u, prefix[u], 0)
    loop = DraftLoop(dv, tv, 3, 4, w.model.vocab, "stochastic", seed=5)
    for u in range(3):
        loop.start_user(u, prefix[u], 20 + u)
    for v in (dv, tv):
        spoiled(v, w.model)
    tv.user_adapter(1, 1)
    r = loop.round(0, np.zeros(3, np.int32), L, 0)
    assert r.token[1] == -1 and r.token[0] >= 0 and r.token[2] >= 0
    assert dv.user_state(1) == tv.user_state(1) == (prefix[1], 21)
    for u in (0, 2):
        assert dv.user_state(u) == tv.user_state(u) == (prefix[u] + 1 + r.n_acc[u], r.token[u])
    tv.user_adapter(1, -1)
    dv.user_adapter(1, 1)
    before = [dv.user_state(u) for u in range(3)]
    with pytest.raises(RuntimeError, match=r"users \[1\]"):
        loop.round(0, np.zeros(3, np.int32), L, 1)
    assert [dv.user_state(u) for u in range(3)] == before == [tv.user_state(u) for u in range(3)]
    dv.user_adapter(1, -1)
    r = loop.round(0, np.zeros(3, np.int32), L, 2)
    assert np.all(r.token >= 0)
    # a user without a token has emitted none
    tv.user_adapter(1, 1)
    gv = GpuVerify(tv, [0, 0, 0], L, w.model.vocab, q_sigma=1.0, commit=False, record=True)
    n = gv(0, 0)
    rec = gv.records[0]
    assert rec.token[1] == -1 and n == rec.n_acc[0] + rec.n_acc[2] + 2
    dv.close()
    tv.close()
