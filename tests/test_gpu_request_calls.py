"""Context-free calls as a server makes them: adapters applied on two streams at
once, and top-k followed by top-p of what it leaves, in two calls."""
import numpy as np
import pytest
import torch

from paper_2604_20919_amd import sdverify as sv
from test_gpu_lora import apply, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [90, 1300])
def test_adapters_on_two_streams_at_once(T):
    """Calls that overlap, each with a workspace of its own, give the bits that
    each gives alone."""
    cs = [make(T, 1024, [512, 64], 16, 6, planes=2, seed=s) for s in (3, 4)]
    alone = [apply(c) for c in cs]
    args, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in cs:
        w = sv.make_lora(c["a"].cuda(), c["b"].cuda(), c["scale"].cuda(), c["segs"])
        outs = [torch.empty_like(c["y"], device="cuda") for _ in range(8)]
        args.append((w, torch.from_numpy(c["ids"]).cuda(), c["x"].cuda(), c["y"].cuda(), outs,
                     torch.empty(sv.sd_lora_query_size(w, T), dtype=torch.uint8, device="cuda"), c["x_lo"].cuda()))
    torch.cuda.synchronize()
    for i in range(8):
        for (w, ids, x, y, outs, ws, lo), s in zip(args, streams):
            sv.sd_lora_apply(w, ids, x, y, outs[i], ws, x_lo=lo, stream=s)
    torch.cuda.synchronize()
    for a, ref in zip(args, alone):
        assert all(torch.equal(o.cpu(), ref) for o in a[4])


@pytest.mark.parametrize("V,k,p,T", [(5003, 50, 0.9, 1.0), (151936, 50, 0.9, 0.8), (32003, 200, 0.5, 1.3)])
def test_top_k_and_then_top_p_of_the_rest(V, k, p, T):
    """The order of servers that renormalise after top-k: a call with
    temperature and top_k, and a second one with top_p on its rows.

    The first call's rows are rounded to fp32, 2^-24 of logarithms up to 20: the
    weights of the second are off by 2^-20 at most, their sums over k tokens by
    less than 2^-20 of the sum.  The inputs keep ten times that away from a border."""
    n = 24
    r = np.random.default_rng(V + k)
    z = (r.standard_normal((n, V)) * r.uniform(1.0, 3.5, (n, 1))).astype(np.float32)
    u = r.random(n).astype(np.float32)
    dev = lambda x, d=torch.float32: torch.full((n,), x, dtype=d, device="cuda")
    zd, rows = torch.from_numpy(z).cuda(), torch.empty((n, V), device="cuda")
    ws = torch.empty(sv.sd_filter_query_size(n, V), dtype=torch.uint8, device="cuda")
    token, kept = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    both = torch.empty_like(kept)
    ud = torch.from_numpy(u).cuda()
    sv.sd_filter_logits(zd, rows, ws, temperature=dev(T), top_k=dev(k, torch.int32))
    sv.sd_sample_filtered(rows, ud, token, ws, top_p=dev(p), kept=kept)
    sv.sd_sample_filtered(zd, ud, torch.empty_like(token), ws, temperature=dev(T), top_k=dev(k, torch.int32), top_p=dev(p),
                          kept=both)
    torch.cuda.synchronize()
    fewer = 0
    for i in range(n):
        order = np.argsort(-z[i].astype(np.float64), kind="stable")[:k]
        w = np.exp((z[i][order].astype(np.float64) - z[i].max()) / np.float32(T).astype(np.float64))
        before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
        border = float(np.float32(p)) * w.sum()
        count = int(np.searchsorted(before, border, side="left"))
        mine = np.sort(order[:count])
        cum = np.cumsum(np.exp((z[i][mine].astype(np.float64) - z[i].max()) / np.float32(T).astype(np.float64)))
        x = float(u[i]) * cum[-1]
        assert min(np.abs(before - border).min(), np.abs(cum - x).min()) > 10 * 2.0 ** -20 * w.sum(), "input at a border"
        assert int(kept[i]) == count
        assert int(token[i]) == mine[int(np.searchsorted(cum, x, side="right"))]
        fewer += count < int(both[i])
    # each filter on the whole distribution keeps no fewer, and mostly more
    assert torch.all(both >= kept) and fewer > n // 2
