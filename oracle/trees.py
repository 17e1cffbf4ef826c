"""Definitions in 64 bits of trees of drafts: attention over a paged cache, rows
and pages moved in it, the walk along the target's tokens, and the rules on
logits.  Plain numpy, one slot or row at a time; test infrastructure like the
rest of the oracle."""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def path_to(parent, j):
    """Slot j and its ancestors, from slot j on (parents outside 0 .. j-1 end it)."""
    out = [j]
    while 0 <= parent[out[-1]] < out[-1]:
        out.append(int(parent[out[-1]]))
    return out


def users_of(slot_off, prefix, n_slots, max_slots):
    """(first slot, slots, cached tokens) of every user."""
    out = []
    for b in range(len(prefix)):
        s0 = min(max(int(slot_off[b]), 0), n_slots)
        s1 = min(max(int(slot_off[b + 1]), s0), n_slots)
        out.append((s0, min(s1 - s0, max_slots), max(int(prefix[b]), 0)))
    return out


def blocks(pool, layer, head, head_dim):
    """Keys [pages][16][head_dim] and values [pages][head_dim][16] of a pool
    [layers][pages][2][heads][16 * head_dim]."""
    p = pool[layer, :, :, head]
    return p[:, 0].reshape(-1, PAGE, head_dim), p[:, 1].reshape(-1, head_dim, PAGE)


def tree_attention(pool, layer, slot_off, prefix, table, parent, q, scale, n_kv_heads, max_slots):
    """(out, size) [slots][heads][head_dim] in 64 bits, NaN where no user owns the
    slot; size: the same with |value| for value, and the scores' largest sum of
    |products|, what errors are measured by (size, score) per output."""
    T, hq, hd = q.shape
    G = hq // n_kv_heads
    out, size = np.full((T, hq, hd), np.nan), np.zeros((T, hq, hd))
    score = np.zeros((T, hq, 1))
    n_pages = pool.shape[1]
    for b, (s0, n, pre) in enumerate(users_of(slot_off, prefix, T, max_slots)):
        par = [j - 1 for j in range(n)] if parent is None else [int(x) for x in parent[s0:s0 + n]]
        for j in range(n):
            see = list(range(min(pre, PAGE * table.shape[1]))) + sorted(pre + a for a in path_to(par, j))
            see = [p for p in see if p < PAGE * table.shape[1] and 0 <= table[b, p // PAGE] < n_pages]
            if not see:
                out[s0 + j] = 0.0
                continue
            pg, at = np.array([table[b, p // PAGE] for p in see]), np.array(see) % PAGE
            for h in range(hq):
                k, v = blocks(pool, layer, h // G, hd)
                keys, vals = k[pg, at], v[pg, :, at]
                z = scale * (keys @ q[s0 + j, h])
                w = np.exp(z - z.max())
                w /= w.sum()
                out[s0 + j, h] = w @ vals
                size[s0 + j, h] = w @ np.abs(vals)
                score[s0 + j, h] = scale * (np.abs(keys) @ np.abs(q[s0 + j, h])).max()
    return out, size, score


def copy_pages(pool, src, dst):
    out, n = pool.copy(), pool.shape[1]
    for a, b in zip(src, dst):
        if 0 <= a < n and 0 <= b < n:
            out[:, b] = pool[:, a]
    return out


def compact(pool, prefix, table, keep, n_keep, head_dim):
    out, n_pages = pool.copy(), pool.shape[1]

    def place(b, p):
        if not 0 <= p < PAGE * table.shape[1] or not 0 <= table[b, p // PAGE] < n_pages:
            return None
        return table[b, p // PAGE], p % PAGE

    for b in range(len(prefix)):
        pre = max(int(prefix[b]), 0)
        for i in range(min(max(int(n_keep[b]), 0), keep.shape[1])):
            k = int(keep[b, i])
            src, dst = (place(b, pre + k) if k >= 0 else None), place(b, pre + i)
            if src is None or dst is None:
                continue
            shape = pool.shape
            old = pool[:, src[0]].reshape(shape[0], 2, shape[3], -1)
            new = out[:, dst[0]].reshape(shape[0], 2, shape[3], -1)
            new[:, 0, :, dst[1] * head_dim:(dst[1] + 1) * head_dim] = old[:, 0, :, src[1] * head_dim:(src[1] + 1) * head_dim]
            new[:, 1, :, dst[1]::PAGE] = old[:, 1, :, src[1]::PAGE]
            out[:, dst[0]] = new
    return out


def walk(target, drafts, parent):
    """(accepted drafts, final token) of one user: target[j] the target's token
    after slot j, drafts[i] and parent[i] of draft i + 1 (slots; 0 the root)."""
    at, path = 0, []
    while True:
        nxt = [i + 1 for i in range(len(drafts)) if parent[i] == at and drafts[i] == target[at]]
        if not nxt:
            return path, int(target[at])
        at = nxt[0]
        path.append(at)


def adjust_row(z, prompt=(), output=(), repetition=1.0, presence=0.0, frequency=0.0, biases=(), allowed=None):
    """One row of logits under the rules; biases: (token, value) pairs, allowed: bool [V] or None."""
    z = np.asarray(z, np.float64).copy()
    V = z.size
    rep = float(repetition) if repetition > 0 and math.isfinite(repetition) else 1.0
    pres = float(presence) if math.isfinite(presence) else 0.0
    freq = float(frequency) if math.isfinite(frequency) else 0.0
    count = {}
    for t in output:
        if 0 <= t < V:
            count[int(t)] = count.get(int(t), 0) + 1
    with np.errstate(invalid="ignore", over="ignore"):
        for t in set(count) | {int(t) for t in prompt if 0 <= t < V}:
            z[t] = z[t] / rep if z[t] > 0 else z[t] * rep
        for t, c in count.items():
            z[t] -= freq * c + pres
        for t, v in {int(t): v for t, v in biases if 0 <= t < V}.items():
            z[t] += float(v)
    if allowed is not None:
        z[~np.asarray(allowed, bool)] = -np.inf
    return z
