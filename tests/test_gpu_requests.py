"""Users' own sampling options and adapters inside verification passes and decode
steps (sd_user_sampling, sd_adapters_set, sd_user_adapter), and both together.

Adapters: the logits of every user equal those of a torch re-implementation in
float64 whose weights have that user's adapter merged in (W + scale B A).  The
models here stay below 2.3e-4 relative logit error without adapters (bf16
activations as two planes; 1e-5 in fp32); the bounds are ten times that.
Sampling options: the pass's logits equal sd_filter_logits of the logits of a
pass without options bit for bit, and the decisions the oracle sampler's on them."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
import workload as wl
from gpu_harness import assert_decisions, compare_decisions, load_synthetic_kv, logit_rel_err, make_verifier
from oracle import requests as rq
from paper_2604_20919_amd import sdverify as sv
from paper_2604_20919_amd.draft_loop import DraftLoop
from test_gpu_sampler import _case, _sampler_verifier
from test_oracle_forward import torch_verify
from workload.device import DeviceWeights, batch_to_device

pytestmark = pytest.mark.gpu


class Adapters:
    """n adapters beside q, k, v (fused), o and down of every layer, on host and GPU."""

    def __init__(self, m, n, rank, seed, sigma=0.05, targets=("qkv", "o", "down")):
        r = np.random.default_rng(seed)
        dt = torch.float32 if m.dtype == "f32" else torch.bfloat16
        nq, nkv = m.n_q_heads * m.head_dim, m.n_kv_heads * m.head_dim
        self.m, self.segs = m, {"qkv": [nq, nkv, nkv], "o": [m.d_model], "down": [m.d_model]}
        d_in = {"qkv": m.d_model, "o": nq, "down": m.d_ffn}
        self.layers, self.host = [], []
        for _ in range(m.n_layers):
            dev, host = {}, {}
            for t in targets:
                seg = self.segs[t]
                a = torch.from_numpy(r.standard_normal((n, len(seg) * rank, d_in[t])) * sigma).to(dt)
                b = torch.from_numpy(r.standard_normal((n, sum(seg), rank)) * sigma).to(dt)
                sc = torch.from_numpy(r.uniform(0.5, 2.0, n)).float()
                dev[t] = sv.make_lora(a.cuda(), b.cuda(), sc.cuda(), seg)
                host[t] = (a.double().numpy(), b.double().numpy(), sc.double().numpy())
            self.layers.append(dev)
            self.host.append(host)

    def merged(self, i, l, t):
        """scale B A of adapter i at a projection, [d_out][d_in]"""
        a, b, sc = (x[i] for x in self.host[l][t])
        rank, out, c = b.shape[1], np.zeros((b.shape[0], a.shape[1])), 0
        for s, w in enumerate(self.segs[t]):
            out[c:c + w] = sc * (b[c:c + w] @ a[s * rank:(s + 1) * rank])
            c += w
        return out


class Merged:
    """A weight source with adapter i merged into its projections, float64."""

    def __init__(self, ws, ad, i):
        self.ws, self.ad, self.i = ws, ad, i

    def global_(self, kind):
        return self.ws.global_(kind)

    def layer(self, l):
        w = {k: (wl.bf16_to_f32(v) if v.dtype == np.uint16 else v).astype(np.float64)
             for k, v in self.ws.layer(l).items()}
        if self.i >= 0:
            for t in self.ad.host[l]:
                delta = self.ad.merged(self.i, l, t)
                if t == "qkv":
                    nq, nkv = self.ad.segs[t][0], self.ad.segs[t][1]
                    for kind, lo, hi in ((wl.W_Q, 0, nq), (wl.W_K, nq, nq + nkv), (wl.W_V, nq + nkv, nq + 2 * nkv)):
                        w[kind] = w[kind].reshape(hi - lo, -1) + delta[lo:hi]
                else:
                    kind = wl.W_O if t == "o" else wl.W_D
                    w[kind] = w[kind].reshape(delta.shape) + delta
        return w


def reference(w, b, ad, ids):
    """Logits of batch b with each user's adapter merged, user by user."""
    m, ws, out, t = w.model, oracle.WeightSource(w.model, w.seed), [], 0
    toks = b.slot_tokens()
    for i, u in enumerate(b.users):
        n = int(b.n_slots[i])
        kv = oracle.KVSource(m, w.seed, [int(u)], [int(b.prefix_len[i])])
        out.append(torch_verify(m, Merged(ws, ad, ids[i]), kv, [int(b.prefix_len[i])], [n], toks[t:t + n],
                                kv_bf16=m.dtype == "bf16"))
        t += n
    return np.concatenate(out)


def verify(v, w, b, mode="stochastic", seed=3, graph=False, stream=None):
    for i, u in enumerate(b.users):
        v.reset_user(int(u), int(b.prefix_len[i]), int(b.root[i]))
    drafts, q, au = batch_to_device(b)
    torch.cuda.synchronize()
    v.verify(0, w.assign, w.draft_len, drafts, q, mode, seed, 0, au, stream=stream, graph=graph)
    lg = v.logits(0, b.T).cpu().numpy()
    acc, tok = v.accept(0, w.n_users)
    torch.cuda.synchronize()
    return lg, acc, tok


def context(model, prefix, L, seed, **kw):
    w = wl.custom_workload(model, prefix, L, seed=seed)
    dw = DeviceWeights(w.model, w.seed)
    v = make_verifier(w, dw, extra_ctx=32, **kw)
    load_synthetic_kv(v, w)
    return w, dw, v


@pytest.mark.parametrize("model,prefix,L,ids", [
    ("tiny", [0, 17, 64, 5], [1, 3, 2, 4], [0, -1, 2, 0]),
    ("tiny-qknorm", [9, 33], [2, 2], [1, 1]),
    ("tiny-bf16", [12], [3], [1]),                                        # few-slot products
    ("tiny-bf16", [40, 300, 0, 17, 5], [1, 7, 3, 5, 2], [0, 1, -1, 2, 1]),
    ("tiny-bf16", [20] * 10, [11, 9, 12, 7, 10, 8, 12, 12, 5, 9], [0, 1, 2, -1, 0, 1, 2, -1, 2, 0]),
    ("tiny-bf16", [8] * 25, [11] * 25, [i % 4 - 1 for i in range(25)]),   # 300 slots: two slot groups
])
def test_logits_with_adapters(model, prefix, L, ids):
    w, dw, v = context(model, prefix, L, seed=61)
    b = w.batch(0)
    plain, acc0, tok0 = verify(v, w, b)
    ad = Adapters(w.model, 3, 8, seed=5)
    v.set_adapters(ad.layers)
    for u, a in zip(b.users, ids):
        v.user_adapter(int(u), a)
    got, _, _ = verify(v, w, b)
    ref = reference(w, b, ad, ids)
    err = logit_rel_err(got, ref)
    assert err.max() < (1e-4 if w.model.dtype == "f32" else 2.3e-3), err.max()
    # slots without adapter are what they were, the others are not
    mine = np.repeat(np.asarray(ids) >= 0, b.n_slots)
    assert np.array_equal(got[~mine], plain[~mine])
    assert logit_rel_err(plain[mine], ref[mine]).min() > 0.02
    # and taking the adapters away brings everything back
    v.set_adapters(None)
    back, acc1, tok1 = verify(v, w, b)
    assert np.array_equal(back, plain) and np.array_equal(acc0, acc1) and np.array_equal(tok0, tok1)
    v.close()


def test_adapters_of_high_rank_over_many_slots():
    """396 slots and three adapters of rank 64: the adapters' 128-row kernels."""
    ids = [i % 4 - 1 for i in range(33)]
    w, dw, v = context("tiny-bf16", [8] * 33, [11] * 33, seed=63)
    b = w.batch(0)
    plain, _, _ = verify(v, w, b)
    ad = Adapters(w.model, 3, 64, seed=5, sigma=0.03)
    v.set_adapters(ad.layers)
    for u, a in zip(b.users, ids):
        v.user_adapter(int(u), a)
    got, _, _ = verify(v, w, b)
    err = logit_rel_err(got, reference(w, b, ad, ids))
    assert err.max() < 2.3e-3, err.max()
    mine = np.repeat(np.asarray(ids) >= 0, b.n_slots)
    assert np.array_equal(got[~mine], plain[~mine])
    st = torch.cuda.Stream()
    for rep in range(3):
        again, _, _ = verify(v, w, b, graph=True, stream=st)
        assert np.array_equal(again, got), rep
    v.close()


@pytest.mark.parametrize("target", ["qkv", "o", "down"])
def test_adapters_beside_one_projection(target):
    w, dw, v = context("tiny-bf16", [30, 4], [4, 2], seed=67)
    b = w.batch(0)
    ad = Adapters(w.model, 2, 5, seed=7, targets=(target,))
    v.set_adapters(ad.layers)
    for u in range(2):
        v.user_adapter(u, 1 - u)
    got, _, _ = verify(v, w, b)
    err = logit_rel_err(got, reference(w, b, ad, [1, 0]))
    assert err.max() < 2.3e-3, err.max()
    v.close()


def test_adapted_caches_are_read_back():
    """Committed rounds with an adapter: the keys and values a user leaves are
    those of its adapted projections (a verify after a commit equals one pass
    over the same tokens)."""
    w, dw, v = context("tiny", [10], [4], seed=71)
    ad = Adapters(w.model, 2, 4, seed=9)
    v.set_adapters(ad.layers)
    v.user_adapter(0, 1)
    toks = wl._ints(9, 71, 5, 0, w.model.vocab - 1).astype(np.int32)
    run = lambda d, commit: (v.verify(0, [0], [len(d)], torch.from_numpy(np.ascontiguousarray(d)).cuda(), None, "force"),
                             v.logits(0, len(d) + 1).cpu().numpy(), v.accept(0, 1, commit=commit))[1]
    v.reset_user(0, 10, int(toks[0]))
    run(toks[1:4], True)
    v.reset_user(0, 14, int(toks[4]))
    second = run(toks[5:9], False)
    ws = oracle.WeightSource(w.model, w.seed)
    kv = oracle.KVSource(w.model, w.seed, [0], [10])
    ref = torch_verify(w.model, Merged(ws, ad, 1), kv, [10], [9], toks)
    assert logit_rel_err(second, ref[4:]).max() < 1e-4
    v.close()


OPTIONS = [(0.7, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (1.3, 20, 1.0, 0.05), (0.0, 0, 1.0, 0.0), (1.0, 0, 0.5, 0.0),
           (0.6, 7, 0.95, 0.2)]


def filtered(logits, opts, slots):
    """The rows of a batch filtered on the GPU by the context-free call."""
    t, k, p, m = (np.repeat([o[i] for o in opts], slots) for i in range(4))
    z = torch.from_numpy(np.ascontiguousarray(logits)).cuda()
    out = torch.empty_like(z)
    ws = torch.empty(sv.sd_filter_query_size(*z.shape), dtype=torch.uint8, device="cuda")
    dev = lambda a, d: torch.from_numpy(a.astype(d)).cuda()
    sv.sd_filter_logits(z, out, ws, dev(t, np.float32), dev(k, np.int32), dev(p, np.float32), dev(m, np.float32))
    torch.cuda.synchronize()
    return out.cpu().numpy()


@pytest.mark.parametrize("model,graph", [("tiny", False), ("tiny-bf16", False), ("tiny-bf16", True)])
def test_verify_with_sampling_options(model, graph):
    prefix, L = [40, 300, 0, 17, 5, 9], [1, 7, 3, 5, 2, 4]
    w, dw, v = context(model, prefix, L, seed=73)
    b = w.batch(0)
    s = torch.cuda.Stream() if graph else None
    raw, acc0, tok0 = verify(v, w, b, graph=graph, stream=s)
    for rep in range(3):
        opts = OPTIONS[rep:] + OPTIONS[:rep]
        for u, o in zip(b.users, opts):
            v.user_sampling(int(u), *o)
        lg, acc, tok = verify(v, w, b, graph=graph, stream=s)
        assert np.array_equal(lg, filtered(raw, opts, b.n_slots))
        ref = oracle.sample("stochastic", b.users, b.draft_len, lg, b.drafts, b.q, b.accept_u, 3, 0)
        chk = compare_decisions(acc[b.users], tok[b.users], ref, b.draft_len, drafts=b.drafts)
        assert_decisions(chk, f"options, {model}, {rep}", end_to_end=False)
        # every token is one of those its filters keep
        for i, u in enumerate(b.users):
            row = int(b.n_slots[:i].sum()) + int(acc[u])
            _, keep, _ = rq.filter_row(raw[row], *opts[i])
            assert keep[tok[u]]
    # greedy and teacher-forced passes take no notice of options
    g1 = verify(v, w, b, "greedy")
    for u in b.users:
        v.user_sampling(int(u))
    g0 = verify(v, w, b, "greedy")
    assert all(np.array_equal(x, y) for x, y in zip(g0, g1))
    raw2, acc2, tok2 = verify(v, w, b, graph=graph, stream=s)
    assert np.array_equal(raw, raw2) and np.array_equal(acc0, acc2) and np.array_equal(tok0, tok2)
    v.close()


@pytest.mark.parametrize("V", [1024, 151936])
def test_sample_logits_with_sampling_options(V):
    Ls = [1, 4, 2, 8, 3, 5]
    logits, q, drafts, au, users = _case(V, Ls, "stochastic", 77, True)
    v = _sampler_verifier(V, 6, 8, sum(Ls) + 6)
    slots = np.asarray(Ls) + 1
    for u, o in zip(users, OPTIONS):
        v.user_sampling(int(u), *o)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    z = dev(logits)
    v.sample(0, np.zeros(6, np.int32), Ls, dev(drafts), dev(q), z, "stochastic", seed=5, round_=1, accept_u=dev(au))
    acc, tok = v.accept(0, 6)
    assert np.array_equal(z.cpu().numpy(), logits)  # the caller's rows stay as they are
    lg = filtered(logits, OPTIONS, slots)
    ref = oracle.sample("stochastic", users, Ls, lg, drafts, q, au, 5, 1)
    assert_decisions(compare_decisions(acc, tok, ref, Ls, drafts=drafts), f"sample options V={V}", end_to_end=False)
    v.close()


def test_decode_step_with_sampling_options():
    """probs rows are the filtered distribution and the token one of its tokens."""
    prefix = [0, 17, 64, 129, 300, 7]
    w, dw, v = context("tiny-bf16", prefix, [4] * 6, seed=79)
    V = w.model.vocab
    for u in range(6):
        v.reset_user(u, prefix[u], 50 + u)
    probs = torch.zeros((6, V), device="cuda")
    a = np.zeros(6, np.int32)
    v.draft(0, a, "stochastic", seed=2, probs=probs)
    raw = v.logits(0, 6).cpu().numpy()
    v.accept(0, 6)
    for u, o in enumerate(OPTIONS):
        v.user_sampling(u, *o)
    for rnd in range(4):
        v.draft(0, a, "stochastic", seed=2, round_=rnd, probs=probs)
        lg = v.logits(0, 6).cpu().numpy()
        _, tok = v.accept(0, 6)
        p = probs.cpu().numpy().astype(np.float64)
        assert np.array_equal(lg, filtered(raw, OPTIONS, np.ones(6, int)))
        for u, o in enumerate(OPTIONS):
            lw, keep, _ = rq.filter_row(raw[u], *o)
            ref = np.exp(lw) / np.exp(lw).sum()
            assert np.all((p[u] > 0) == keep) and keep[tok[u]]
            assert np.all(np.abs(p[u] - ref) <= 2e-5 * ref + 1e-12)
    v.close()


def test_options_and_adapters_together_in_the_drafting_loop():
    """Drafting and target contexts hold the same model, adapters and options:
    every draft is accepted over committed rounds, in passes whose users differ
    in both (accept uniforms of 0.5 stay off the u ~ p/q window)."""
    prefix, L = [33, 7, 90, 128], [3, 1, 4, 2]
    w, dw, dv = context("tiny-bf16", prefix, L, seed=83, max_batch_tokens=len(prefix) * 5)
    tv = make_verifier(w, dw, extra_ctx=32, max_batch_tokens=len(prefix) * 5)
    load_synthetic_kv(tv, w)
    ad = Adapters(w.model, 3, 16, seed=11)
    loop = DraftLoop(dv, tv, 4, max(L), w.model.vocab, "stochastic", seed=5)
    roots = wl._ints(4, 83, 78, 0, w.model.vocab - 1)
    for v in (dv, tv):
        v.set_adapters(ad.layers)
    for u, a in enumerate((2, -1, 0, 1)):
        loop.start_user(u, prefix[u], int(roots[u]))
        loop.user_sampling(u, *OPTIONS[(0, 2, 3, 4)[u]])
        dv.user_adapter(u, a)
        tv.user_adapter(u, a)
    half = torch.full((sum(L),), 0.5, device="cuda")
    orig = tv.verify
    tv.verify = lambda *a, **k: orig(*a, **{**k, "accept_u": half})
    for rnd in range(4):
        r = loop.round(0, np.zeros(4, np.int32), L, rnd)
        assert np.array_equal(r.n_acc, np.asarray(L)), (rnd, r.n_acc)
        for u in range(4):
            assert dv.user_state(u) == tv.user_state(u)
    dv.close()
    tv.close()


def test_refusals():
    w, dw, v = context("tiny-bf16", [9, 3], [2, 2], seed=89)
    bad = [(-1.0, 0, 1.0, 0.0), (float("nan"), 0, 1.0, 0.0), (float("inf"), 0, 1.0, 0.0), (1.0, -1, 1.0, 0.0),
           (1.0, 0, 0.0, 0.0), (1.0, 0, 1.5, 0.0), (1.0, 0, float("nan"), 0.0), (1.0, 0, 1.0, -0.1), (1.0, 0, 1.0, 1.1)]

    def refused(status, f, *a):
        with pytest.raises(sv.SdError) as e:
            f(*a)
        assert e.value.status == status
    for o in bad:
        refused(sv.SD_EINVAL, v.user_sampling, 0, *o)
    refused(sv.SD_EINVAL, v.user_sampling, 2, 1.0)
    refused(sv.SD_EINVAL, v.user_adapter, 0, 0)  # none set
    ad = Adapters(w.model, 2, 4, seed=1)
    other = Adapters(wl.MODELS["tiny"], 2, 4, seed=1)
    v.set_adapters(ad.layers)
    refused(sv.SD_EINVAL, v.user_adapter, 0, 2)
    refused(sv.SD_EINVAL, v.user_adapter, 0, -2)
    refused(sv.SD_EINVAL, v.user_adapter, 2, 0)
    v.user_adapter(0, 1)
    refused(sv.SD_EINVAL, v.set_adapters, other.layers)  # another model's: refused, the set stays
    mixed = [dict(ad.layers[0]), dict(ad.layers[1])]
    mixed[1]["o"] = Adapters(w.model, 3, 4, seed=1).layers[1]["o"]
    refused(sv.SD_EINVAL, v.set_adapters, mixed)
    with pytest.raises(ValueError):
        v.set_adapters(ad.layers[:1])
    b = w.batch(0)
    drafts, q, au = batch_to_device(b)
    for i, u in enumerate(b.users):
        v.reset_user(int(u), int(b.prefix_len[i]), int(b.root[i]))
    v.verify(0, w.assign, w.draft_len, drafts, q, "stochastic")
    refused(sv.SD_ESTATE, v.user_sampling, 0, 0.5)
    refused(sv.SD_ESTATE, v.user_adapter, 0, -1)
    refused(sv.SD_ESTATE, v.set_adapters, None)
    v.accept(0, 2)
    v.set_adapters(None)
    v.close()


def test_sparse_draft_rows_with_options_and_adapters():
    """Sparse draft rows against the dense rows they stand for, in a pass whose
    users have options and adapters: the same decisions."""
    prefix, L = [12, 70, 5], [3, 5, 2]
    w, dw, v = context("tiny-bf16", prefix, L, seed=91)
    b = w.batch(0)
    sp = wl.sparsify(b, 16, 7)
    q = oracle.expand_sparse_q(sp.idx, sp.val, sp.rest, w.model.vocab)
    ad = Adapters(w.model, 2, 128, seed=3, sigma=0.02)
    v.set_adapters(ad.layers)
    for u, (o, a) in enumerate(zip(OPTIONS, (1, -1, 0))):
        v.user_sampling(u, *o)
        v.user_adapter(u, a)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    drafts, idx, val, rest, dense = dev(b.drafts), dev(sp.idx), dev(sp.val), dev(sp.rest), dev(q)
    for seed in range(4):
        for i, u in enumerate(b.users):
            v.reset_user(int(u), int(b.prefix_len[i]), int(b.root[i]))
        v.verify_sparse(0, w.assign, w.draft_len, drafts, idx, val, rest, seed=seed)
        a = v.accept(0, 3)
        v.verify(0, w.assign, w.draft_len, drafts, dense, seed=seed)
        d = v.accept(0, 3)
        assert np.array_equal(a[0], d[0]) and np.array_equal(a[1], d[1])
    v.close()


def test_two_batches_at_once():
    """Two pending batches on two streams, users of both with options and adapters,
    give what each gives alone."""
    prefix, L = [30, 5, 90, 17, 64, 2], [4, 2, 6, 3, 5, 1]
    w = wl.custom_workload("tiny-bf16", prefix, L, seed=97, assign=[0, 1, 0, 1, 0, 1])
    dw = DeviceWeights(w.model, w.seed)
    v = make_verifier(w, dw, extra_ctx=32)
    load_synthetic_kv(v, w)
    ad = Adapters(w.model, 3, 12, seed=13)
    v.set_adapters(ad.layers)
    ins = []
    for n in range(2):
        b = w.batch(n)
        ins.append((b, batch_to_device(b)))
        for i, u in enumerate(b.users):
            v.reset_user(int(u), int(b.prefix_len[i]), int(b.root[i]))
    for u in range(6):
        v.user_sampling(u, *OPTIONS[u])
        v.user_adapter(u, u % 4 - 1)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()

    def go(n):
        b, (d, q, au) = ins[n]
        v.verify(n, w.assign, w.draft_len, d, q, "stochastic", seed=4, accept_u=au, stream=streams[n])

    alone = []
    for n in range(2):
        go(n)
        lg = v.logits(n, ins[n][0].T, streams[n])
        acc, tok = v.accept(n, 6)
        torch.cuda.synchronize()
        alone.append((lg.cpu().numpy(), acc, tok))
    for rep in range(4):
        go(0)
        go(1)
        for n in (1, 0):
            lg = v.logits(n, ins[n][0].T, streams[n])
            acc, tok = v.accept(n, 6)
            torch.cuda.synchronize()
            assert np.array_equal(lg.cpu().numpy(), alone[n][0])
            assert np.array_equal(acc, alone[n][1]) and np.array_equal(tok, alone[n][2])
    v.close()


def test_options_of_a_vocabulary_beyond_the_filters():
    v = _sampler_verifier(sv.SD_FILTER_MAX_VOCAB + 4, 1, 1, 2)
    with pytest.raises(sv.SdError) as e:
        v.user_sampling(0, 0.5)
    assert e.value.status == sv.SD_ELIMIT
    v.close()
    v = _sampler_verifier(sv.SD_FILTER_MAX_VOCAB, 1, 1, 2)
    v.user_sampling(0, 0.5, top_k=1 << 40)
    v.close()
