"""Users without sampling options beside users that have some: their decisions,
tokens and distributions are those of a pass without such users, bit for bit,
not-a-numbers and infinities among their logits included."""
import numpy as np
import pytest
import torch

import oracle
import workload as wl
from gpu_harness import assert_decisions, compare_decisions
from paper_2604_20919_amd import sdverify as sv
from test_gpu_requests import OPTIONS, context, filtered
from test_gpu_sampler import _case, _sampler_verifier
from workload.device import batch_to_device

pytestmark = pytest.mark.gpu

dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
FREE = [1, 3, 4]  # users without options


def set_options(v, on, n=6):
    for u in range(n):
        v.user_sampling(u, *(OPTIONS[(0, 2, 5)[u % 3]] if on and u not in FREE else ()))


@pytest.mark.parametrize("model,logits_out", [("tiny", sv.SD_LOGITS_ALL), ("tiny-bf16", sv.SD_LOGITS_AS_NEEDED),
                                              ("tiny-bf16", sv.SD_LOGITS_UNFUSED)])
@pytest.mark.parametrize("how", ["plain", "graph", "sparse"])
def test_decisions_beside_users_with_options(model, logits_out, how):
    prefix, L = [40, 300, 0, 17, 5, 9], [1, 7, 3, 5, 2, 4]
    w, dw, v = context(model, prefix, L, seed=109, logits_out=logits_out)
    b = w.batch(0)
    drafts, q, au = batch_to_device(b)
    sp = wl.sparsify(b, 16, 7)
    sparse = [dev(x) for x in (sp.idx, sp.val, sp.rest)]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()

    def go(seed):
        for i, u in enumerate(b.users):
            v.reset_user(int(u), int(b.prefix_len[i]), int(b.root[i]))
        if how == "sparse":
            v.verify_sparse(0, w.assign, w.draft_len, drafts, *sparse, seed=seed, stream=st)
        else:
            v.verify(0, w.assign, w.draft_len, drafts, q, "stochastic", seed, 0, None, stream=st, graph=how == "graph")
        lg = v.logits(0, b.T, st)
        acc, tok = v.accept(0, 6)
        torch.cuda.synchronize()
        return lg.cpu().numpy(), acc, tok

    alone = [go(seed) for seed in range(25)]
    set_options(v, True)
    opts = [OPTIONS[1] if u in FREE else OPTIONS[(0, 2, 5)[u % 3]] for u in range(6)]
    moved = False
    for seed, (raw, acc0, tok0) in enumerate(alone):
        lg, acc, tok = go(seed)
        assert np.array_equal(acc[FREE], acc0[FREE]) and np.array_equal(tok[FREE], tok0[FREE]), seed
        assert np.array_equal(lg, filtered(raw, opts, b.n_slots))
        moved |= not np.array_equal(tok, tok0)
    assert moved
    v.close()


@pytest.mark.parametrize("model", ["tiny", "tiny-bf16"])
def test_distributions_beside_users_with_options(model):
    prefix = [0, 17, 64, 129, 300, 7]
    w, dw, v = context(model, prefix, [4] * 6, seed=113)
    V = w.model.vocab
    for u in range(6):
        v.reset_user(u, prefix[u], 50 + u)
    a = np.zeros(6, np.int32)
    got = []
    for on in (False, True):
        set_options(v, on)
        runs = []
        for seed in range(10):
            probs = torch.zeros((6, V), device="cuda")
            v.draft(0, a, "stochastic", seed=seed, probs=probs)
            runs.append((v.accept(0, 6)[1], probs.cpu().numpy()))
        got.append(runs)
    for (tok0, p0), (tok, p) in zip(*got):
        assert np.array_equal(tok[FREE], tok0[FREE]) and np.array_equal(p[FREE], p0[FREE])
        assert not np.array_equal(p[[0, 2, 5]], p0[[0, 2, 5]])
    v.close()


@pytest.mark.parametrize("V", [1024, 4099, 151936])
def test_caller_logits_beside_users_with_options(V):
    """Caller's logits, three users with options, the others' rows holding
    not-a-numbers and infinities."""
    Ls = [1, 4, 2, 8, 3, 5]
    logits, q, drafts, au, users = _case(V, Ls, "stochastic", 79, True)
    off = np.cumsum([0] + [l + 1 for l in Ls])
    v = _sampler_verifier(V, 6, 8, sum(Ls) + 6)
    for what in (None, np.nan, np.inf, -np.inf):
        z = logits.copy()
        if what is not None:
            z[off[1] + 1, 3] = what
            z[off[3], V - 1] = what
            z[off[4] + 1] = what
        got = []
        for on in (False, True):
            set_options(v, on)
            runs = []
            for seed in range(8):
                zd = dev(z)
                v.sample(0, np.zeros(6, np.int32), Ls, dev(drafts), dev(q), zd, "stochastic", seed=seed, round_=1,
                         accept_u=dev(au))
                runs.append(v.accept(0, 6))
                assert np.array_equal(zd.cpu().numpy(), z, equal_nan=True)
            got.append(runs)
        for (acc0, tok0), (acc, tok) in zip(*got):
            assert np.array_equal(acc[FREE], acc0[FREE]) and np.array_equal(tok[FREE], tok0[FREE]), what
    opts = [OPTIONS[1] if u in FREE else OPTIONS[(0, 2, 5)[u % 3]] for u in range(6)]
    lg = filtered(logits, opts, np.asarray(Ls) + 1)
    ref = oracle.sample("stochastic", users, Ls, lg, drafts, q, au, 5, 1)
    v.sample(0, np.zeros(6, np.int32), Ls, dev(drafts), dev(q), dev(logits), "stochastic", seed=5, round_=1, accept_u=dev(au))
    acc, tok = v.accept(0, 6)
    assert_decisions(compare_decisions(acc, tok, ref, Ls, drafts=drafts), f"mixed options V={V}", end_to_end=False)
    v.close()
