"""Rules on the caller's logits (sd_batch_rules with sd_sample_logits): users whose contexts
are full are sampled like any other, for such a call takes no pages and writes no cache."""
import numpy as np
import pytest
import torch

import oracle
from paper_2604_20919_amd import sdverify as sv
from test_gpu_sampler import _case, _sampler_verifier
from test_gpu_tree_pass import BatchRules, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["greedy", "stochastic"])
def test_users_near_the_end_of_their_contexts(mode):
    Ls = [1, 4, 2, 8]
    logits, q, drafts, au, users = _case(1024, Ls, mode, 81, True)
    v = _sampler_verifier(1024, 4, 8, sum(Ls) + 4)
    prefix = [0, 62, 0, 60]  # of 64: no room for a pass over the slots of the second and the fourth
    for u in range(4):
        v.reset_user(u, prefix[u], 11 * u)
    a, z = np.zeros(4, np.int32), torch.from_numpy(logits).cuda()
    R = BatchRules(1024, np.repeat(range(4), np.array(Ls) + 1), 9)
    toks = np.concatenate([[11 * u] + list(d) for u, d in enumerate(np.split(drafts, np.cumsum(Ls)[:-1]))])
    j = np.concatenate([np.arange(n + 1) for n in Ls])
    want = R.apply(logits, toks, np.where(j > 0, np.arange(j.size) - 1, -1))
    pages = [list(v.user_pages(u)) for u in range(4)]
    for rules, rows in ((None, logits), (R.make(), want)):
        if rules is not None:
            v.batch_rules(0, rules)
        v.sample(0, a, Ls, dev(drafts), dev(q, np.float32), z, mode, 5, 1, dev(au, np.float32))
        acc, tok = v.accept(0, 4)
        ref = oracle.sample(mode, users, Ls, rows, drafts, q, au, 5, 1)
        assert np.array_equal(acc, ref["n_acc"]) and np.array_equal(tok, ref["token"])
    # a pass over them is refused as ever, with rules and without
    for rules in (None, R.make()):
        v.batch_rules(0, rules)
        with pytest.raises(sv.SdError) as e:
            v.verify(0, a, Ls, dev(drafts), dev(q, np.float32), mode, 5, 1)
        assert e.value.status == sv.SD_EINVAL
    assert pages == [list(v.user_pages(u)) for u in range(4)]
    v.close()
