"""Timed cases of the verification of drafted trees and of what surrounds it: attention of a tree's
slots over the paged cache, pages copied and accepted rows moved together in it, and the rules
(penalties, biases, grammar masks) that a request's logits pass before a token is taken.  Each case is
one call through the public entry points, or the same result in elementary torch operations.

A case is a dict of plain values:
  call   "tree"     attention of users' drafted trees over their cached contexts: sd_tree_attention
         "copy"     pages of a cache copied in all layers (a user forked): sd_kv_copy_pages
         "compact"  rows of the accepted drafts moved together in all layers: sd_kv_compact
         "rules"    logits under penalties, biases and masks: sd_adjust_logits
  tree: users, slots and ctx as ranges "lo,hi" (slots of a user: its root and drafts), hq, hkv, hd,
  dtype, planes (2: queries as a high and a low bf16 plane, as inside the verify pass), lens (seed of
  the users' sizes, trees and pages)
  copy: pages, layers, hkv, hd, dtype;  compact: users, slots and keep as ranges, layers, hkv, hd, dtype
  rules: rows, vocab, dtype, users (rows of a user follow each other and share its history), hist as a
  range, biases (listed tokens a user), masks (a grammar mask a row), pad (elements between rows)

Queries and cached rows are N(0, 1), as after the QK norm.  Pages are taken in random order.  Trees
are drawn breadth-first with a few children a node.  Histories repeat tokens as text does (Zipf).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

VOCAB = 151936
PAGE = 16
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _tree(name, users, slots, ctx, hq, hkv, hd, lens, dtype="bf16", planes=1):
    return {"name": name, "call": "tree", "users": users, "slots": slots, "ctx": ctx, "hq": hq, "hkv": hkv, "hd": hd,
            "dtype": dtype, "planes": planes, "lens": lens}


def _copy(name, pages, layers, hkv, hd, lens, dtype="bf16"):
    return {"name": name, "call": "copy", "pages": pages, "layers": layers, "hkv": hkv, "hd": hd, "dtype": dtype,
            "lens": lens}


def _compact(name, users, slots, keep, layers, hkv, hd, lens, dtype="bf16"):
    return {"name": name, "call": "compact", "users": users, "slots": slots, "keep": keep, "layers": layers, "hkv": hkv,
            "hd": hd, "dtype": dtype, "lens": lens}


def _rules(name, rows, users, hist, lens, vocab=VOCAB, dtype="f32", biases=0, masks=False, pad=0):
    return {"name": name, "call": "rules", "rows": rows, "users": users, "hist": hist, "vocab": vocab, "dtype": dtype,
            "biases": biases, "masks": masks, "pad": pad, "lens": lens}


def listed():
    return [
        # one device's tree of a few drafts, a short chat, one layer of the small model
        _tree("tree-1-1.7b", 1, "8,8", "200,200", 16, 8, 128, 1),
        # the repository's headline batch: 32 users of 2 to 13 slots, queries in two planes
        _tree("tree-ragged32-32b", 32, "2,13", "256,4096", 64, 8, 128, 2, planes=2),
        # wide trees over long contexts: bound by the products, not by the cache
        _tree("tree-wide16-32b", 16, "64,64", "1024,8192", 64, 8, 128, 3),
        # one token of one user over a very long cache
        _tree("tree-decode-long", 1, "1,1", "131072,131072", 32, 4, 64, 4),
        # a fp32 model of odd contexts
        _tree("tree-f32", 6, "3,17", "63,900", 12, 4, 64, 5, dtype="f32"),
        # a short prompt forked on the small model
        _copy("copy-3-1.7b", 3, 28, 8, 128, 6),
        # a prompt of 1280 tokens forked on the large model
        _copy("copy-80-32b", 80, 64, 8, 128, 7),
        # one user's accepted path, small model
        _compact("compact-1-1.7b", 1, "8,8", "3,3", 28, 8, 128, 8),
        # the accepted paths of 32 users' trees, large model
        _compact("compact-32-32b", 32, "24,64", "1,8", 64, 8, 128, 9),
        # one token of a user with penalties
        _rules("rules-1", 1, 1, "2000,2000", 10),
        # the headline's 229 slots, every user with penalties and a few biases
        _rules("rules-229", 229, 32, "256,4096", 11, biases=40),
        # the widest batch in bf16 logits, a grammar mask a slot, rows padded apart
        _rules("rules-416-masks", 416, 40, "100,9000", 12, dtype="bf16", biases=300, masks=True, pad=24),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    call = rng.choice(["tree", "tree", "tree", "rules", "rules", "copy", "compact"])
    lens = rng.randrange(1 << 20)
    if call == "tree":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        f32 = dtype == "f32"
        hkv = rng.choice([1, 2, 3, 4, 8])
        hq = hkv * rng.choice([1, 2, 4, 5, 8])
        hd = rng.choice([64, 128])
        slots = _log_int(rng, 1, 24 if f32 else 64)
        ctx = _log_int(rng, 1, 2000 if f32 else 60000)
        # rows times context within the widest listed case
        most = (2e7 if f32 else 1.5e8) / (slots * (ctx + slots) * hq)
        users = min(_log_int(rng, 1, 64), max(1, int(most)))
        return {"call": call, "users": users, "slots": "%d,%d" % (max(1, slots // rng.randint(1, 4)), slots),
                "ctx": "%d,%d" % (ctx // rng.randint(1, 8), ctx), "hq": hq, "hkv": hkv, "hd": hd, "dtype": dtype,
                "planes": 1 if f32 else rng.choice([1, 2]), "lens": lens}
    if call == "rules":
        vocab = rng.choice([VOCAB, rng.randint(30000, 160000), _log_int(rng, 900, 160000)])
        rows = _log_int(rng, 1, 416)
        hist = _log_int(rng, 1, 9000)
        return {"call": call, "rows": rows, "users": rng.randint(1, min(rows, 64)), "vocab": vocab,
                "hist": "%d,%d" % (hist // rng.randint(1, 8), hist), "dtype": rng.choice(["f32", "f32", "bf16"]),
                "biases": rng.choice([0, 0, 3, 40, 300]), "masks": rng.random() < 0.5,
                "pad": rng.choice([0, 0, rng.randint(1, 64)]), "lens": lens}
    hkv, hd = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    layers, dtype = rng.randint(1, 64), rng.choice(["bf16", "bf16", "f32"])
    if call == "copy":
        page = layers * hkv * hd * SIZE[dtype]
        return {"call": call, "pages": min(_log_int(rng, 1, 400), max(1, 64 * 80 * 8 * 128 * 2 // page)), "layers": layers,
                "hkv": hkv, "hd": hd, "dtype": dtype, "lens": lens}
    slots = rng.randint(2, 64)
    keep = rng.randint(1, max(1, min(12, slots // 2)))
    return {"call": call, "users": rng.randint(1, 32 if dtype == "bf16" else 16), "slots": "%d,%d" % (2 * keep, max(slots, 2 * keep)),
            "keep": "%d,%d" % (rng.randint(0, keep), keep), "layers": layers, "hkv": hkv, "hd": hd, "dtype": dtype,
            "lens": lens}


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _range(text):
    lo, hi = text.split(",")
    return int(lo), int(hi)


def _parents(r, n):
    """A tree of n slots, breadth-first: each draft below one of the last few nodes of its level or the one before."""
    return [-1] + [max(0, (j - 1) // r.choice([1, 2, 2, 3])) for j in range(1, n)]


def _users(case):
    """The users' slots, prefixes, parents and pages (from the case alone, as a server's users keep theirs)."""
    r = random.Random(case["lens"])
    slots = [r.randint(*_range(case["slots"])) for _ in range(case["users"])]
    prefix = [r.randint(*_range(case["ctx"])) for _ in slots] if "ctx" in case else [r.randint(0, 60) for _ in slots]
    parent = [p for n in slots for p in _parents(r, n)]
    counts = [-(-(p + n) // PAGE) for p, n in zip(prefix, slots)]
    pages = list(range(sum(counts) + 3))
    r.shuffle(pages)
    table, at = [], 0
    for c in counts:
        table.append(pages[at:at + c] + [0] * (max(counts) - c))
        at += c
    return slots, prefix, parent, table, len(pages)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(sizes):
    return [sum(sizes[:i]) for i in range(len(sizes) + 1)]


def _pool(g, dtype, layers, pages, hkv, hd):
    """[layer][page][K | V][kv_head] blocks; K blocks [16][hd], V blocks [hd][16]."""
    pool = torch.empty((layers, pages, 2, hkv, PAGE * hd), dtype=DT[dtype], device="cuda")
    return pool.normal_(generator=g)


def _kept(case, slots):
    """Accepted slots of each user: its root, then drafts further down its list than the path is long."""
    r = random.Random(case["lens"] + 1)
    keep = []
    for n in slots:
        k = r.randint(*_range(case["keep"]))
        k = min(k, n // 2) if n > 1 else min(k, 1)
        keep.append(([0] + sorted(r.sample(range(k, n), k - 1))) if k else [])
    return keep


def _layout(case):
    """The rows' users and trees, the users' options (plain values, from the case alone)."""
    r = random.Random(case["lens"])
    cuts = sorted(r.sample(range(1, case["rows"]), case["users"] - 1))
    ends = cuts + [case["rows"]]
    sizes = [b - a for a, b in zip([0] + cuts, ends)]
    users = []
    for n in sizes:
        h = r.randint(*_range(case["hist"]))
        users.append({"rows": n, "hist": h, "prompt": r.randint(0, h), "parents": _parents(r, n),
                      "repetition": r.choice([1.0, 1.05, 1.2]), "presence": r.choice([0.0, 0.5, 1.0]),
                      "frequency": r.choice([0.0, 0.2, 0.7])})
    return users


def _prepare_tree(case, seed):
    g, dt = _gen(seed, 1), DT[case["dtype"]]
    slots, prefix, parent, table, n_pages = _users(case)
    T, hq, hd = sum(slots), case["hq"], case["hd"]
    q = torch.randn((T, hq, hd), generator=g, device="cuda")
    hi = q.to(dt)
    return {"case": case, "pool": _pool(g, case["dtype"], 1, n_pages, case["hkv"], hd), "q": hi,
            "q_lo": (q - hi.float()).to(dt) if case["planes"] == 2 else None, "out": torch.empty_like(hi),
            "slot_off": _ints(_offsets(slots)), "prefix": _ints(prefix), "parent": _ints(parent), "table": _ints(table),
            "most": max(slots), "longest": max(p + n for p, n in zip(prefix, slots))}


def _prepare_copy(case, seed):
    g, r = _gen(seed, 2), random.Random(case["lens"])
    n = case["pages"]
    pages = list(range(2 * n))
    r.shuffle(pages)
    return {"case": case, "pool": _pool(g, case["dtype"], case["layers"], 2 * n, case["hkv"], case["hd"]),
            "src": _ints(pages[:n]), "dst": _ints(pages[n:])}


def _prepare_compact(case, seed):
    slots, prefix, _, table, n_pages = _users(case)
    keep = _kept(case, slots)
    most = max(1, max(len(k) for k in keep))
    return {"case": case, "pool": _pool(_gen(seed, 3), case["dtype"], case["layers"], n_pages, case["hkv"], case["hd"]),
            "prefix": _ints(prefix), "table": _ints(table), "keep": _ints([k + [-1] * (most - len(k)) for k in keep]),
            "n_keep": _ints([len(k) for k in keep])}


def _prepare_rules(case, seed):
    g, V, n = _gen(seed, 4), case["vocab"], case["rows"]
    users = _layout(case)
    total = sum(u["hist"] for u in users)
    zipf = torch.rand(max(total, 1), generator=g, device="cuda")
    order = torch.randperm(V, generator=g, device="cuda").int()
    tokens = order[(torch.pow(float(V), zipf) - 1).long().clamp(0, V - 1)]
    begin = _offsets([u["hist"] for u in users])
    rows = [(i, u) for i, u in enumerate(users) for _ in range(u["rows"])]
    first = _offsets([u["rows"] for u in users])
    parent = [p if p < 0 else first[i] + p for i, u in enumerate(users) for p in u["parents"]]
    floats = lambda key: torch.tensor([u[key] for _, u in rows], dtype=torch.float32, device="cuda")  # noqa: E731
    buf = torch.randn((n, V + case["pad"]), generator=g, device="cuda") * 2.5
    s = {"case": case, "logits": buf.to(DT[case["dtype"]])[:, :V], "tokens": tokens,
         "hist": _ints([[begin[i], begin[i] + u["prompt"], begin[i] + u["hist"]] for i, u in rows]),
         "repetition": floats("repetition"), "presence": floats("presence"), "frequency": floats("frequency"),
         "row_token": torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32), "row_parent": _ints(parent),
         "bias_token": None, "bias_value": None, "bias": None, "mask": None, "mask_row": None}
    k = min(case["biases"], V)
    if k:
        # each user's tokens are distinct, as in a request's map
        s["bias_token"] = torch.cat([torch.randperm(V, generator=g, device="cuda")[:k] for _ in users]).int()
        s["bias_value"] = torch.randn(k * len(users), generator=g, device="cuda") * 4.0
        s["bias"] = _ints([[k * i, k * (i + 1)] for i, _ in rows])
    if case["masks"]:
        # grammars allow few tokens at some positions and most of them at others
        words = torch.randint(-2**31, 2**31, (3, n, -(-V // 32)), generator=g, device="cuda").int()
        few = (torch.arange(n, device="cuda") % 3 == 0).unsqueeze(1)
        s["mask"] = torch.where(few, words[0] & words[1] & words[2], words[0] | words[1] | words[2])
        s["mask_row"] = _ints(list(range(n)))
    s["out"] = torch.empty((n, V), dtype=torch.float32, device="cuda")
    return s


def prepare(case, seed):
    return {"tree": _prepare_tree, "copy": _prepare_copy, "compact": _prepare_compact, "rules": _prepare_rules}[case["call"]](case, seed)


def _closure(parent):
    """[..., n, n]: whether column j is row i or an ancestor of it, for parents [..., n] (negative: none)."""
    n = parent.shape[-1]
    at = torch.arange(n, device=parent.device)
    reach = ((parent.unsqueeze(-1) == at) | (at.unsqueeze(-1) == at)).float()
    for _ in range(max(1, (n - 1).bit_length())):
        reach = (reach @ reach > 0).float()
    return reach > 0


def _tree_plain(s):
    case, dev = s["case"], s["q"].device
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    B, S, C, G = case["users"], s["most"], s["longest"], hq // hkv
    q = s["q"].float() if s["q_lo"] is None else s["q"].float() + s["q_lo"].float()
    off, prefix = s["slot_off"].long(), s["prefix"].long()
    slots = off[1:] - off[:-1]
    j = torch.arange(S, device=dev)
    mine = j < slots.unsqueeze(1)
    row = (off[:-1].unsqueeze(1) + j).clamp(max=q.shape[0] - 1)
    tok = torch.arange(C, device=dev)
    live = tok < (prefix + slots).unsqueeze(1)
    page = s["table"].long()[:, tok // PAGE]
    blocks = s["pool"][0]
    n_pages = blocks.shape[0]
    k = blocks[:, 0].reshape(n_pages, hkv, PAGE, hd)[page, :, tok % PAGE].float()
    v = blocks[:, 1].reshape(n_pages, hkv, hd, PAGE)[page, :, :, tok % PAGE].float()
    seen = _closure(torch.where(mine, s["parent"].long()[row], -1))
    rel = tok - prefix.unsqueeze(1)
    below = (rel < 0).unsqueeze(1) | seen.gather(2, rel.clamp(0, S - 1).unsqueeze(1).expand(B, S, C))
    below = below & live.unsqueeze(1)
    qs = q[row].reshape(B, S, hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, S * G, hd)
    z = qs @ k.permute(0, 2, 3, 1).contiguous() * (1.0 / math.sqrt(hd))
    z = z.masked_fill(~below.repeat_interleave(G, dim=1).unsqueeze(1), -math.inf)
    w = torch.exp(z - z.amax(dim=3, keepdim=True))
    o = (w @ v.permute(0, 2, 1, 3).contiguous()) / w.sum(dim=3, keepdim=True)
    o = o.reshape(B, hkv, S, G, hd).permute(0, 2, 1, 3, 4).reshape(B, S, hq, hd)
    return o[mine].to(s["q"].dtype)


def _compact_plain(s):
    case, pool = s["case"], s["pool"]
    hkv, hd = case["hkv"], case["hd"]
    at = torch.arange(s["keep"].shape[1], device=pool.device)
    user, i = (at < s["n_keep"].unsqueeze(1)).nonzero(as_tuple=True)
    src = s["prefix"].long()[user] + s["keep"].long()[user, i]
    dst = s["prefix"].long()[user] + i
    sp, dp = s["table"].long()[user, src // PAGE], s["table"].long()[user, dst // PAGE]
    k = pool[:, :, 0].unflatten(-1, (PAGE, hd))
    v = pool[:, :, 1].unflatten(-1, (hd, PAGE))
    kr, vr = k[:, sp, :, src % PAGE], v[:, sp, :, :, src % PAGE]
    k[:, dp, :, dst % PAGE] = kr
    v[:, dp, :, :, dst % PAGE] = vr
    return pool


def _rules_plain(s):
    z = s["logits"].float()
    n, V = z.shape
    hist = s["hist"].long()
    size = hist[:, 2] - hist[:, 0]
    row = torch.repeat_interleave(torch.arange(n, device=z.device), size)
    at = torch.arange(row.numel(), device=z.device) - (torch.cumsum(size, 0) - size)[row] + hist[row, 0]
    tok, prompt = s["tokens"].long()[at], at < hist[row, 1]
    anc_row, anc = _closure(s["row_parent"].long()).nonzero(as_tuple=True)
    flat = lambda r, t: torch.bincount(r * V + t, minlength=n * V).reshape(n, V)  # noqa: E731
    count = flat(torch.cat([row[~prompt], anc_row]), torch.cat([tok[~prompt], s["row_token"].long()[anc]]))
    seen = (count > 0) | (flat(row[prompt], tok[prompt]) > 0)
    rep = s["repetition"].unsqueeze(1)
    y = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z)
    y = torch.where(count > 0, y - (s["frequency"].unsqueeze(1) * count.float() + s["presence"].unsqueeze(1)), y)
    if s["bias"] is not None:
        span = s["bias"].long()
        m = span[:, 1] - span[:, 0]
        r = torch.repeat_interleave(torch.arange(n, device=z.device), m)
        e = torch.arange(r.numel(), device=z.device) - (torch.cumsum(m, 0) - m)[r] + span[r, 0]
        y[r, s["bias_token"].long()[e]] += s["bias_value"][e]
    if s["mask"] is not None:
        k = torch.arange(V, device=z.device)
        y = torch.where((s["mask"][s["mask_row"].long()][:, k // 32] >> (k % 32)) & 1 == 1, y, -math.inf)
    return y


def run(s):
    call = s["case"]["call"]
    if own:
        from paper_2604_20919_amd import sdverify as sv
        if "plan" not in s:  # what a server keeps from call to call
            if call == "rules":
                s["plan"] = sv.make_logit_rules(
                    s["case"]["rows"], s["case"]["vocab"], tokens=s["tokens"], hist=s["hist"], repetition=s["repetition"],
                    presence=s["presence"], frequency=s["frequency"], row_token=s["row_token"], row_parent=s["row_parent"],
                    bias_token=s["bias_token"], bias_value=s["bias_value"], bias=s["bias"], mask=s["mask"],
                    mask_row=s["mask_row"])
            else:
                shape = s["pool"].shape
                s["plan"] = sv.make_kv_pool(s["pool"], shape[0], shape[1], s["case"]["hkv"], s["case"]["hd"])
            if call == "tree":
                s["trees"] = sv.make_tree(s["slot_off"], s["prefix"], s["table"], s["parent"], max_slots=s["most"])
                s["ws"] = torch.empty(sv.sd_tree_query_size(s["plan"], s["trees"], s["case"]["hq"]), dtype=torch.uint8,
                                      device="cuda")
        if call == "tree":
            sv.sd_tree_attention(s["plan"], 0, s["trees"], s["q"], s["out"], s["ws"], q_lo=s["q_lo"])
            return s["out"]
        if call == "copy":
            sv.sd_kv_copy_pages(s["plan"], s["src"], s["dst"])
            return s["pool"]
        if call == "compact":
            sv.sd_kv_compact(s["plan"], s["prefix"], s["table"], s["keep"], s["n_keep"])
            return s["pool"]
        sv.sd_adjust_logits(s["logits"], s["plan"], s["out"])
        return s["out"]
    if call == "tree":
        return _tree_plain(s)
    if call == "copy":
        s["pool"][:, s["dst"].long()] = s["pool"][:, s["src"].long()]
        return s["pool"]
    if call == "compact":
        return _compact_plain(s)
    return _rules_plain(s)


def work(case):
    if case["call"] == "tree":
        slots, prefix, parent, _, _ = _users(case)
        es, T = SIZE[case["dtype"]], sum(slots)
        tokens = sum(slots) + sum(prefix)
        depth, at = [], 0
        for n in slots:
            d = []
            for p in parent[at:at + n]:
                d.append(1 if p < 0 else d[p] + 1)
            depth += d
            at += n
        seen = sum(n * p for n, p in zip(slots, prefix)) + sum(depth)
        return {"bytes": tokens * 2 * case["hkv"] * case["hd"] * es + T * case["hq"] * case["hd"] * es * (case["planes"] + 1),
                "flops": 4 * case["hq"] * case["hd"] * seen}
    if case["call"] in ("copy", "compact"):
        row = 2 * case["layers"] * case["hkv"] * case["hd"] * SIZE[case["dtype"]]
        if case["call"] == "copy":
            return {"bytes": 2 * case["pages"] * PAGE * row, "flops": 0}
        # rows that stay where they are move nothing
        moved = sum(a != i for k in _kept(case, _users(case)[0]) for i, a in enumerate(k))
        return {"bytes": max(1, 2 * moved * row), "flops": 0}
    n = case["rows"] * case["vocab"]
    users = _layout(case)
    lists = 4 * sum(u["hist"] for u in users) + 8 * min(case["biases"], case["vocab"]) * len(users)
    return {"bytes": n * (SIZE[case["dtype"]] + 4) + (n // 8 if case["masks"] else 0) + lists + 32 * case["rows"], "flops": n}


def exact(case, seed):
    if case["call"] in ("copy", "compact"):
        return None  # nothing is computed
    s = prepare(case, seed)
    if case["call"] == "tree":
        slots, prefix, parent, table, n_pages = _users(case)
        hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
        G = hq // hkv
        q = s["q"].double() + (0.0 if s["q_lo"] is None else s["q_lo"].double())
        out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        at = 0
        for u, (n, p) in enumerate(zip(slots, prefix)):
            ids = table[u][:-(-(p + n) // PAGE)]
            blocks = s["pool"][0, ids]
            keys = blocks[:, 0].reshape(len(ids), hkv, PAGE, hd).permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :p + n].double()
            values = blocks[:, 1].reshape(len(ids), hkv, hd, PAGE).permute(1, 0, 3, 2).reshape(hkv, -1, hd)[:, :p + n].double()
            allowed = torch.zeros((n, p + n), dtype=torch.bool)
            allowed[:, :p] = True
            for j in range(n):
                a = j
                while a >= 0:
                    allowed[j, p + a] = True
                    a = parent[at + a]
            allowed = allowed.cuda()
            for h in range(hq):
                z = q[at:at + n, h] @ keys[h // G].t().contiguous() / math.sqrt(hd)
                w = torch.softmax(z.masked_fill(~allowed, -math.inf), dim=1)
                out[at:at + n, h] = w @ values[h // G]
            at += n
        return out
    z = s["logits"].float().cpu().numpy().astype(np.float64)
    n, V = z.shape
    get = lambda key: None if s[key] is None else s[key].cpu().numpy()  # noqa: E731
    tokens, hist, row_token, row_parent = get("tokens"), get("hist"), get("row_token"), get("row_parent")
    rep, pres, freq = (get(k).astype(np.float64) for k in ("repetition", "presence", "frequency"))
    bt, bv, br, mask = get("bias_token"), get("bias_value"), get("bias"), get("mask")
    for i in range(n):
        b, e, f = (int(x) for x in hist[i])
        path, a = [], i
        while a >= 0:
            path.append(int(row_token[a]))
            a = int(row_parent[a])
        made = np.concatenate([tokens[e:f], np.array(path, dtype=tokens.dtype)])
        got, times = np.unique(made, return_counts=True)
        both = np.union1d(got, tokens[b:e])
        z[i, both] = np.where(z[i, both] > 0, z[i, both] / rep[i], z[i, both] * rep[i])
        z[i, got] -= freq[i] * times + pres[i]
        if br is not None:
            z[i, bt[br[i, 0]:br[i, 1]]] += bv[br[i, 0]:br[i, 1]].astype(np.float64)
        if mask is not None:
            bits = np.unpackbits(mask[i].view(np.uint8), bitorder="little")[:V]
            z[i, bits == 0] = -np.inf
    return z
