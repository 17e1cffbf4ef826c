"""Timed cases of what a request brings of its own to a shared batch: its sampling options and its
low-rank adapter.  Each case is one call through the public entry points, or the same result in
elementary torch operations.

A case is a dict of plain values:
  call    "sample"  a token a row from filtered logits and given uniforms: sd_sample_filtered
          "filter"  the filtered rows themselves, which accept/resample reads: sd_filter_logits
          "lora"    adapters of many requests beside a shared projection: sd_lora_apply
  sample, filter: rows, vocab, dtype of the logits, pad (elements between rows), lens (seed of the
  rows' options), plain (temperature alone, no filter)
  lora: rows, d_in, q/k/v or one segment of outputs ("segs"), rank, adapters, dtype, y_dtype, planes
  (2: x as a high and a low bf16 plane, the products' input in the verify pass), per (rows that
  follow each other with one adapter: a user's slots), none (share of users without adapter)

Rows' options are drawn per row as a server meets them: a few greedy rows, temperatures 0.6 to 1.3,
top-k, top-p and min-p each on some rows.  Logits are normal with a row's own width (1.43 is that of
the repository's random-init 32B shape, wider ones stand for trained models) and a few outstanding
tokens.  Adapters are N(0, 0.02), activations N(0, 1), the shared projection's outputs N(0, 1).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

VOCAB = 151936
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _rows(name, call, rows, vocab, dtype, lens, pad=0, plain=False):
    return {"name": name, "call": call, "rows": rows, "vocab": vocab, "dtype": dtype, "pad": pad, "lens": lens,
            "plain": plain}


def _lora(name, rows, d_in, segs, rank, adapters, per, lens, dtype="bf16", y_dtype="f32", planes=1, none=0.0):
    return {"name": name, "call": "lora", "rows": rows, "d_in": d_in, "segs": segs, "rank": rank, "adapters": adapters,
            "per": per, "lens": lens, "dtype": dtype, "y_dtype": y_dtype, "planes": planes, "none": none}


def listed():
    return [
        # a device drafting one token for itself: the smallest call
        _rows("sample-1", "sample", 1, VOCAB, "f32", 1),
        # one decode step of 32 users, each with its own options
        _rows("sample-32", "sample", 32, VOCAB, "f32", 2),
        # a small odd vocabulary in bf16, rows padded apart
        _rows("sample-130-bf16", "sample", 130, 32003, "bf16", 3, pad=29),
        # temperature alone on a busy server: no filter at all
        _rows("sample-256-plain", "sample", 256, VOCAB, "f32", 4, plain=True),
        # the widest batch of slots the library verifies
        _rows("sample-416", "sample", 416, VOCAB, "f32", 5),
        # six users of seven drafts: the paper's standard verification
        _rows("filter-48", "filter", 48, VOCAB, "f32", 6),
        # the repository's headline batch, every slot's logits filtered before accept/resample
        _rows("filter-229", "filter", 229, VOCAB, "f32", 7),
        # a device's own adapter beside the fused q, k, v of the small model, one token
        _lora("lora-1-qkv-1.7b", 1, 2048, "2048,1024,1024", 16, 4, 1, 1),
        # 16 users of 5 slots beside the large model's down projection, input in two planes
        _lora("lora-80-down-32b", 80, 25600, "5120", 32, 16, 5, 2, planes=2),
        # the headline's 229 slots beside the large model's q, k, v, two planes, some users without adapter
        _lora("lora-229-qkv-32b", 229, 5120, "8192,1024,1024", 16, 32, 7, 3, planes=2, none=0.2),
        # a fp32 adapter of odd sizes
        _lora("lora-45-f32-odd", 45, 1000, "1328", 12, 6, 3, 4, dtype="f32"),
        # prompts of four adapters entering side by side, outputs in bf16
        _lora("lora-8192-o-32b", 8192, 8192, "5120", 64, 4, 1500, 5, y_dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["sample", "sample", "filter", "lora", "lora"])
    lens = rng.randrange(1 << 20)
    if call == "lora":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        f32 = dtype == "f32"
        # one size in four odd, which leaves rows without the alignment that wide loads need
        even = rng.random() < 0.75
        size = lambda lo, hi: 16 * rng.randint(lo, hi) if even else rng.randint(16 * lo, 16 * hi)  # noqa: E731
        q = size(8, 320)
        segs = rng.choice(["%d" % q, "%d,%d,%d" % (q, size(4, 64), size(4, 64))])
        rows = _log_int(rng, 1, 400 if f32 else 4000)
        return {"call": call, "rows": rows, "d_in": size(8, 512), "segs": segs,
                "rank": rng.choice([1, 4, 8, 12, 16, 24, 32, 64]), "adapters": _log_int(rng, 1, 32 if rows <= 512 else 4),
                "per": _log_int(rng, 1, 64) if rows <= 512 else rng.randint(200, 2000), "lens": lens, "dtype": dtype,
                "y_dtype": rng.choice(["f32", "f32", "bf16"]), "planes": 1 if f32 else rng.choice([1, 2]),
                "none": rng.choice([0.0, 0.25])}
    vocab = rng.choice([VOCAB, rng.randint(30000, 160000), _log_int(rng, 900, 160000)])
    return {"call": call, "rows": _log_int(rng, 1, 400 if call == "sample" else 220), "vocab": vocab,
            "dtype": rng.choice(["f32", "f32", "bf16"]), "pad": rng.choice([0, 0, rng.randint(1, 64)]), "lens": lens,
            "plain": rng.random() < 0.15}


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _options(case):
    """The rows' options: plain lists, from the case alone (a server's users keep theirs)."""
    r = random.Random(case["lens"])
    temp, top_k, top_p, min_p = [], [], [], []
    for _ in range(case["rows"]):
        temp.append(0.0 if r.random() < 0.06 else r.uniform(0.6, 1.3))
        top_k.append(r.choice([20, 50, 200, 1000]) if r.random() < 0.4 else 0)
        top_p.append(r.uniform(0.7, 0.99) if r.random() < 0.6 else 1.0)
        min_p.append(r.uniform(0.01, 0.1) if r.random() < 0.25 else 0.0)
    if case["plain"]:
        temp = [max(t, 0.5) for t in temp]
    return temp, top_k, top_p, min_p


def _owners(case):
    """The adapter of each row: users' slots follow each other, each user with one adapter or none."""
    r = random.Random(case["lens"])
    ids = []
    while len(ids) < case["rows"]:
        n = r.randint(max(1, case["per"] // 2), case["per"] + case["per"] // 2)
        a = -1 if r.random() < case["none"] else r.randrange(case["adapters"])
        ids += [a] * min(n, case["rows"] - len(ids))
    return ids


def prepare(case, seed):
    if case["call"] == "lora":
        g = _gen(seed, 7)
        dt, T, R = DT[case["dtype"]], case["rows"], case["rank"]
        segs = [int(s) for s in case["segs"].split(",")]
        d_out, n = sum(segs), case["adapters"]
        x = torch.randn((T, case["d_in"]), generator=g, device="cuda")
        hi = x.to(dt)
        s = {"case": case, "segs": segs, "x": hi,
             "x_lo": (x - hi.float()).to(dt) if case["planes"] == 2 else None,
             "a": (torch.randn((n, len(segs) * R, case["d_in"]), generator=g, device="cuda") * 0.02).to(dt),
             "b": (torch.randn((n, d_out, R), generator=g, device="cuda") * 0.02).to(dt),
             "scale": torch.rand(n, generator=g, device="cuda") + 0.5,
             "ids": torch.tensor(_owners(case), dtype=torch.int32, device="cuda"),
             "y": torch.randn((T, d_out), generator=g, device="cuda").to(DT[case["y_dtype"]])}
        s["out"] = torch.empty_like(s["y"])
        return s
    g = _gen(seed, 3)
    n, V = case["rows"], case["vocab"]
    buf = torch.randn((n, V + case["pad"]), generator=g, device="cuda")
    buf *= 1.0 + 2.5 * torch.rand((n, 1), generator=g, device="cuda")
    at = torch.randint(0, V, (n, 32), generator=g, device="cuda")
    buf.scatter_add_(1, at, 4.0 * torch.rand((n, 32), generator=g, device="cuda"))
    z = buf.to(DT[case["dtype"]])[:, :V]
    temp, top_k, top_p, min_p = _options(case)
    s = {"case": case, "logits": z, "temperature": torch.tensor(temp, dtype=torch.float32, device="cuda"),
         "top_k": None if case["plain"] else torch.tensor(top_k, dtype=torch.int32, device="cuda"),
         "top_p": None if case["plain"] else torch.tensor(top_p, dtype=torch.float32, device="cuda"),
         "min_p": None if case["plain"] else torch.tensor(min_p, dtype=torch.float32, device="cuda"),
         "u": torch.rand(n, generator=g, device="cuda")}
    s["kept"] = torch.empty(n, dtype=torch.int32, device="cuda")
    if case["call"] == "sample":
        s["token"] = torch.empty(n, dtype=torch.int32, device="cuda")
        s["prob"] = torch.empty(n, dtype=torch.float32, device="cuda")
    else:
        s["out"] = torch.empty((n, V), dtype=torch.float32, device="cuda")
    return s


def _filtered(s):
    """(z - max) / T in 64 bits, the weights exp of it, and the kept tokens, in index order.  Sums are
    in 64 bits: a token next to a border is kept or not by them."""
    z = s["logits"].float()
    n, V = z.shape
    order, at = torch.sort(z, dim=1, descending=True, stable=True)
    t = s["temperature"].double().unsqueeze(1)
    greedy = t == 0
    y = (order.double() - order[:, :1].double()) / torch.where(greedy, 1.0, t)
    w = torch.exp(y)
    rank = torch.arange(V, device=z.device)
    keep = ~greedy | (rank == 0)
    if s["top_k"] is not None:
        k = s["top_k"].unsqueeze(1)
        keep = keep & ((k <= 0) | (rank < k))
        p = s["top_p"].double().unsqueeze(1)
        cum = torch.cumsum(w, dim=1)
        keep = keep & ((p >= 1) | (cum - w < p * cum[:, -1:]))
        keep = keep & (w >= s["min_p"].double().unsqueeze(1))
        keep = keep | (rank == 0)
    back = torch.empty_like(at).scatter_(1, at, rank.expand(n, V))
    return y.gather(1, back), keep.gather(1, back)


def _lora_plain(s):
    ids, segs, R = s["ids"].long(), s["segs"], s["case"]["rank"]
    x = s["x"].float() if s["x_lo"] is None else s["x"].float() + s["x_lo"].float()
    n, T = s["a"].shape[0], x.shape[0]
    h = (x @ s["a"].float().reshape(-1, x.shape[1]).t()).reshape(T, n, len(segs), R)
    mine = (ids.unsqueeze(1) == torch.arange(n, device=ids.device)).float() * s["scale"]
    h = h * mine.reshape(T, n, 1, 1)
    ends = np.cumsum([0] + segs)
    b = s["b"].float()
    delta = [h[:, :, i].reshape(T, -1) @ b[:, ends[i]:ends[i + 1]].permute(0, 2, 1).reshape(n * R, -1)
             for i in range(len(segs))]
    return (s["y"].float() + torch.cat(delta, dim=1)).to(s["y"].dtype)


def run(s):
    case = s["case"]
    if own:
        from paper_2604_20919_amd import sdverify as sv
        if "ws" not in s:  # what a server keeps from call to call
            if case["call"] == "lora":
                s["set"] = sv.make_lora(s["a"], s["b"], s["scale"], segs=s["segs"])
                size = sv.sd_lora_query_size(s["set"], case["rows"])
            else:
                size = sv.sd_filter_query_size(case["rows"], case["vocab"])
            s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        if case["call"] == "lora":
            sv.sd_lora_apply(s["set"], s["ids"], s["x"], s["y"], s["out"], s["ws"], x_lo=s["x_lo"])
            return s["out"]
        if case["call"] == "sample":
            sv.sd_sample_filtered(s["logits"], s["u"], s["token"], s["ws"], temperature=s["temperature"],
                                  top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"], kept=s["kept"])
            return {"token": s["token"], "prob": s["prob"], "kept": s["kept"]}
        sv.sd_filter_logits(s["logits"], s["out"], s["ws"], temperature=s["temperature"], top_k=s["top_k"],
                            top_p=s["top_p"], min_p=s["min_p"], kept=s["kept"])
        return {"out": s["out"], "kept": s["kept"]}
    if case["call"] == "lora":
        return _lora_plain(s)
    y, keep = _filtered(s)
    kept = keep.sum(dim=1, dtype=torch.int32)
    if case["call"] == "filter":
        return {"out": torch.where(keep, y, -math.inf).float(), "kept": kept}
    w = torch.where(keep, torch.exp(y), 0.0)
    cum = torch.cumsum(w, dim=1)
    token = (cum <= s["u"].double().unsqueeze(1) * cum[:, -1:]).sum(dim=1, keepdim=True).clamp(max=w.shape[1] - 1)
    prob = w.gather(1, token) / cum[:, -1:]
    return {"token": token.squeeze(1).int(), "prob": prob.squeeze(1).float(), "kept": kept}


def work(case):
    if case["call"] == "lora":
        segs = [int(v) for v in case["segs"].split(",")]
        T, R, n_seg, d_out = case["rows"], case["rank"], len(segs), sum(segs)
        ids = _owners(case)
        used, live = len(set(ids) - {-1}), sum(i >= 0 for i in ids)
        es, ey = SIZE[case["dtype"]], SIZE[case["y_dtype"]]
        return {"bytes": used * R * (n_seg * case["d_in"] + d_out) * es + live * case["d_in"] * es * case["planes"]
                + 2 * T * d_out * ey + 4 * T,
                "flops": 2 * live * R * (n_seg * case["d_in"] * case["planes"] + d_out)}
    n = case["rows"] * case["vocab"]
    read = n * SIZE[case["dtype"]]
    # one exponential an element: a subtraction, a product and a polynomial
    return {"bytes": read + (12 * case["rows"] if case["call"] == "sample" else 4 * n), "flops": 24 * n}


def exact(case, seed):
    s = prepare(case, seed)
    if case["call"] == "lora":
        x = s["x"].double() + (0.0 if s["x_lo"] is None else s["x_lo"].double())
        y, ids, R = s["y"].double(), _owners(case), case["rank"]
        for a in sorted(set(ids) - {-1}):
            rows = torch.tensor([t for t, i in enumerate(ids) if i == a], device="cuda")
            c = 0
            for i, d in enumerate(s["segs"]):
                h = x[rows] @ s["a"][a, i * R:(i + 1) * R].double().t()
                y[rows, c:c + d] += s["scale"][a].double() * (h @ s["b"][a, c:c + d].double().t())
                c += d
        return y
    z = s["logits"].float().cpu().numpy().astype(np.float64)
    temp, u = s["temperature"].cpu().numpy().astype(np.float64), s["u"].cpu().numpy().astype(np.float64)
    n, V = z.shape
    opts = [None if s[o] is None else s[o].cpu().numpy().astype(np.float64) for o in ("top_k", "top_p", "min_p")]
    kept, token, prob = np.zeros(n, np.int32), np.zeros(n, np.int32), np.zeros(n)
    out = np.full((n, V), -np.inf) if case["call"] == "filter" else None
    for i in range(n):
        order = np.argsort(-z[i], kind="stable")
        count = V
        with np.errstate(divide="ignore"):
            lw = (z[i] - z[i][order[0]]) / temp[i] if temp[i] > 0 else np.where(np.arange(V) == order[0], 0.0, -np.inf)
        wt = np.exp(lw)
        if temp[i] == 0:
            count = 1
        if opts[0] is not None:
            if opts[0][i] > 0:
                count = min(count, int(opts[0][i]))
            if opts[1][i] < 1:
                before = np.concatenate(([0.0], np.cumsum(wt[order])[:-1]))
                count = min(count, int(np.searchsorted(before, opts[1][i] * wt.sum(), side="left")))
            count = min(count, int(np.count_nonzero(wt[order] >= opts[2][i])))
            count = max(count, 1)
        mine = np.sort(order[:count])
        kept[i] = count
        if out is not None:
            out[i, mine] = lw[mine]
            continue
        cum = np.cumsum(wt[mine])
        at = min(int(np.searchsorted(cum, u[i] * cum[-1], side="right")), count - 1)
        token[i], prob[i] = mine[at], wt[mine[at]] / cum[-1]
    return {"out": out, "kept": kept} if out is not None else {"kept": kept, "prob": prob, "token": token}
