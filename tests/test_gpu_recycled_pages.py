"""What a user leaves in its cache pages -- infinities and not-a-numbers of its
own adapter among it -- has no part in another user's attention, nor in its own
once the rows lie past its context."""
import numpy as np
import pytest
import torch

import workload as wl
from gpu_harness import load_synthetic_kv
from paper_2604_20919_amd import sdverify as sv
from test_gpu_requests import Adapters, context, verify

pytestmark = pytest.mark.gpu


def fill(v, w, users, n, commit):
    """A pass of n drafts a user whose keys and values are not-a-numbers."""
    for u in range(w.n_users):
        v.user_adapter(u, 1 if u in users else -1)
    a = np.array([0 if u in users else -1 for u in range(w.n_users)], np.int32)
    d = torch.ones(n * len(users), dtype=torch.int32, device="cuda")
    v.verify(0, a, [n] * w.n_users, d, None, "force")
    acc, _ = v.accept(0, w.n_users, commit=commit)
    assert all(acc[u] == n for u in users)
    for u in users:
        v.user_adapter(u, -1)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("model,prefix,L", [
    ("tiny", [9, 40], [2, 1]),
    ("tiny-bf16", [9, 40], [2, 1]),             # short items: blocks in registers
    ("tiny-bf16", [700, 37, 5], [1, 1, 2]),     # longer ones among them
    ("tiny-bf16", [70, 300, 1], [11, 7, 12]),   # blocks through LDS
])
def test_pages_of_other_users(model, prefix, L, bad):
    w, dw, v = context(model, prefix, L, seed=107, max_draft=20, max_batch_tokens=21 * len(prefix))
    b = w.batch(0)
    clean, acc0, tok0 = verify(v, w, b)
    assert np.isfinite(clean).all()
    ad = Adapters(w.model, 2, 4, seed=3, targets=("qkv",))
    for l in ad.layers:
        l["qkv"].scale[1] = bad
    v.set_adapters(ad.layers)
    everyone = list(range(w.n_users))
    # rows past the context, from a longer pass that was not committed
    fill(v, w, everyone, 20, commit=False)
    lg, acc, tok = verify(v, w, b)
    assert np.array_equal(lg, clean) and np.array_equal(acc, acc0) and np.array_equal(tok, tok0)
    # pages that another user has filled and given back
    fill(v, w, everyone, 20, commit=True)
    for u in everyone:
        sv.sd_user_release(v.ctx, u)
    load_synthetic_kv(v, w)
    lg, acc, tok = verify(v, w, b)
    assert np.array_equal(lg, clean) and np.array_equal(acc, acc0) and np.array_equal(tok, tok0)
    v.close()
