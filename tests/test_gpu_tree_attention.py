"""Attention of trees of drafts over a paged cache (sd_tree_attention) against its
64-bit definition (oracle.trees).

Tolerances, with u = 2^-24, S the largest scale * sum |q k| of a slot's keys and W =
sum of weights * |v|: a score is a sum of head_dim products in fp32, off by at most
2 (head_dim + 12) u S (a factor of 2 for the matrix cores' own order), an exponential
by 2^-21 more, numerator and denominator alike: the weights move by twice that.
The weights of the bf16 path enter the second product as two planes, 2^-17 of each
left out.  Sums over n keys add n u, twice.  The output is rounded once: half a step
of bf16 (2^-8), of two planes (2^-16) or of fp32 (2^-24)."""
import numpy as np
import pytest
import torch

from oracle import trees
from paper_2604_20919_amd import sdverify as sv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def parents(r, n, kind):
    if kind == "chain":
        return [j - 1 for j in range(n)]
    if kind == "flat":
        return ([-1] + [0] * n)[:n]
    if kind == "roots":  # nobody below anybody
        return [-1] * n
    return ([-1] + [int(r.integers(max(0, j - 6), j)) for j in range(1, n)])[:n]


class Case:
    """users: (prefix, slots); everything on host and GPU."""

    def __init__(self, users, dtype="bf16", hd=128, hkv=2, G=4, kind="tree", planes=1, pad=0, seed=0, layers=2, layer=1,
                 max_slots=None, spare_pages=2, spare_slots=0, no_parent=False):
        r = np.random.default_rng(seed)
        self.hd, self.hkv, self.hq, self.layer, self.dtype, self.planes = hd, hkv, hkv * G, layer, dtype, planes
        counts = [-(-(p + n) // 16) for p, n in users]
        n_pages = sum(counts) + spare_pages
        order = r.permutation(n_pages)
        most = max(max(counts), 1)
        self.table = np.zeros((len(users), most), np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = order[at:at + c]
            at += c
        self.prefix = np.array([p for p, _ in users], np.int32)
        self.off = np.concatenate([[0], np.cumsum([n for _, n in users])]).astype(np.int32)
        self.T = int(self.off[-1]) + spare_slots
        self.parent = np.array([p for _, n in users for p in parents(r, n, kind)] + [7] * spare_slots, np.int32)
        self.no_parent = no_parent
        self.max_slots = max_slots or max(max(n for _, n in users), 1)
        g = torch.Generator().manual_seed(seed)
        self.pool = torch.randn((layers, n_pages, 2, hkv, 16 * hd), generator=g).to(DT[dtype])
        q = torch.randn((self.T, self.hq, hd), generator=g)
        self.q = q.to(DT[dtype])
        self.q_lo = (q - self.q.float()).to(DT[dtype]) if planes == 2 else None
        self.pad = pad

    def spread(self, t, fill=float("nan")):
        """[T][hq][hd] with `pad` elements between slots, on the GPU."""
        row = self.hq * self.hd
        buf = torch.full((self.T * (row + self.pad),), fill, dtype=t.dtype, device="cuda")
        v = buf.as_strided(t.shape, (row + self.pad, self.hd, 1))
        v.copy_(t)
        return v

    def to_gpu(self):
        i = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.d_pool = self.pool.cuda()
        self.kv = sv.make_kv_pool(self.d_pool, self.pool.shape[0], self.pool.shape[1], self.hkv, self.hd)
        self.d = [i(self.off), i(self.prefix), i(self.table), None if self.no_parent else i(self.parent)]
        self.tree = sv.make_tree(*self.d, max_slots=self.max_slots, n_slots=self.T)
        self.d_q = self.spread(self.q)
        self.d_lo = None if self.q_lo is None else self.spread(self.q_lo)
        self.out = self.spread(torch.full(self.q.shape, -7.0, dtype=self.q.dtype))
        self.out_lo = self.spread(torch.full(self.q.shape, -7.0, dtype=self.q.dtype)) if self.planes == 2 else None
        self.ws = torch.empty(sv.sd_tree_query_size(self.kv, self.tree, self.hq), dtype=torch.uint8, device="cuda")
        return self

    def call(self, scale=None, stream=None):
        sv.sd_tree_attention(self.kv, self.layer, self.tree, self.d_q, self.out, self.ws, q_lo=self.d_lo, out_lo=self.out_lo,
                             scale=scale, stream=stream)

    def check(self, label, scale=None, out=None, out_lo=None, scores_of=None):
        torch.cuda.synchronize()
        sc = self.hd ** -0.5 if scale is None else scale
        q = self.q.double().numpy() + (0 if self.q_lo is None else self.q_lo.double().numpy())
        with np.errstate(invalid="ignore", over="ignore"):
            ref, size, score = trees.tree_attention(self.pool.double().numpy(), self.layer, self.off, self.prefix, self.table,
                                                    None if self.no_parent else self.parent, q, sc, self.hkv, self.max_slots)
            if scores_of is not None:  # a pool without the keys that weigh nothing: no error of theirs counts
                score = trees.tree_attention(scores_of.double().numpy(), self.layer, self.off, self.prefix, self.table,
                                             None if self.no_parent else self.parent, q, sc, self.hkv, self.max_slots)[2]
        got = (self.out if out is None else out).double().cpu().numpy()
        lo = self.out_lo if out_lo is None else out_lo
        nobody = np.isnan(ref) & (size == 0)
        assert (got[nobody] == -7.0).all(), f"{label}: slots of nobody were written"
        if lo is not None:
            got = np.where(nobody, got, got + lo.double().cpu().numpy())
        n = min(int(self.prefix.max()), 16 * self.table.shape[1]) + self.max_slots  # most keys of a slot
        step = {"f32": 2.0 ** -24, "bf16": 2.0 ** -16 if self.planes == 2 else 2.0 ** -8}[self.dtype]
        tol = size * (4 * (self.hd + 12) * U * score + 2.0 ** -20 + 2 * n * U + (2.0 ** -17 if self.dtype == "bf16" else 0.0))
        tol = tol + step * np.abs(ref)
        mine = ~nobody
        fine = np.isfinite(ref) & mine
        assert np.array_equal(np.isnan(ref[mine]), np.isnan(got[mine])), f"{label}: not-a-numbers"
        bad = mine & ~np.isnan(ref) & ~np.isfinite(ref)
        assert np.array_equal(ref[bad], got[bad]), f"{label}: infinities"
        off = np.abs(got - ref)[fine] / np.maximum(tol[fine], 1e-300)
        off = np.where(np.abs(got - ref)[fine] == 0, 0.0, off)
        print(f"{label}: {int(fine.sum())} outputs, worst {off.max() if off.size else 0:.3f} of the tolerance", flush=True)
        assert off.size == 0 or off.max() <= 1.0, f"{label}: {off.max()} times the tolerance"


@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("f32", 128), ("f32", 6), ("f32", 36), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("kind", ["tree", "chain", "flat", "roots"])
def test_ragged_users(dtype, hd, kind):
    users = [(0, 1), (1, 3), (15, 2), (16, 1), (17, 9), (31, 5), (33, 17), (64, 4), (300, 12), (0, 7), (5, 0), (127, 33)]
    c = Case(users, dtype, hd, kind=kind, seed=hd + len(kind)).to_gpu()
    c.call()
    c.check(f"{dtype} {hd} {kind}")


@pytest.mark.parametrize("hd", [2, 34, 64, 70, 100, 128])
@pytest.mark.parametrize("users", [[(0, 1), (1, 9), (63, 2), (64, 3), (200, 17), (255, 1)], [(700, 4)] + [(90, 5)] * 70,
                                   [(1100, 3), (0, 2)]])
def test_fp32_contexts(hd, users):
    """Short contexts, many workgroups, and neither."""
    c = Case(users, "f32", hd, 2, 5, seed=hd).to_gpu()
    c.call()
    c.check(f"f32 {hd}")


@pytest.mark.parametrize("hkv,G", [(1, 1), (1, 5), (3, 1), (2, 8), (1, 16), (1, 40), (4, 3), (1, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_layouts(hkv, G, dtype):
    c = Case([(40, 6), (3, 1), (130, 11)], dtype, 64, hkv, G, seed=G).to_gpu()
    c.call()
    c.check(f"{dtype} {hkv}x{G}")


@pytest.mark.parametrize("planes,pad", [(2, 0), (1, 8), (2, 40)])
@pytest.mark.parametrize("hd", [64, 128])
def test_planes_and_strides(planes, pad, hd):
    c = Case([(100, 13), (0, 4), (513, 5), (30, 30)], "bf16", hd, planes=planes, pad=pad, seed=pad).to_gpu()
    c.call()
    c.check(f"{planes} planes, pad {pad}")


def test_fp32_strides_of_any_size():
    c = Case([(100, 13), (0, 4)], "f32", 10, 1, 3, pad=7, seed=5).to_gpu()
    c.call()
    c.check("fp32 pad 7")


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 200, 255, 256])
@pytest.mark.parametrize("prefix", [0, 13, 96])
def test_tree_sizes(n, prefix):
    c = Case([(prefix, n), (7, 2)], "bf16", 64, 1, 2, seed=n + prefix).to_gpu()
    c.call()
    c.check(f"{n} slots after {prefix}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_contexts(dtype):
    c = Case([(5000, 2), (0, 1), (9999, 1), (1500, 20)], dtype, 64, 1, 2, seed=3, layers=1, layer=0).to_gpu()
    c.call()
    c.check(f"{dtype} long")


def test_one_user_among_many():
    c = Case([(int(p), 1) for p in np.random.default_rng(1).integers(0, 90, 300)] + [(2500, 3)], "bf16", 64, 1, 2, seed=4).to_gpu()
    c.call()
    c.check("301 users")


def test_scale_and_chains_without_parents():
    c = Case([(50, 9), (3, 3)], "bf16", 128, no_parent=True, seed=6).to_gpu()
    c.call(scale=0.5)
    c.check("chain, scale 0.5", scale=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slots_of_nobody_stay_and_wrong_offsets_are_clamped(dtype):
    c = Case([(20, 3), (40, 4), (60, 5)], dtype, 64, spare_slots=5, seed=8)
    c.off = np.array([-4, 3, 900, 2], np.int32)  # users of 3, 14 (4 counted) and no slots
    c.max_slots = 4
    c.to_gpu().call()
    c.check("clamped")
    assert (c.out[7:].float() == -7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_and_parents_outside_mean_nothing(dtype):
    c = Case([(100, 6), (40, 5), (20, 3), (3, 2)], dtype, 64, seed=9)
    c.table[0, 2], c.table[0, 4] = -1, c.pool.shape[1]
    c.table[1, :] = 1 << 30  # nothing of this user
    c.prefix[3] = -9         # counts as 0
    c.parent[:6] = [3, 1, 0, -8, 99, 4]
    c.to_gpu().call()
    c.check("outside")
    assert (c.out[6:11].float() == 0).all()


def test_positions_beyond_the_page_table():
    c = Case([(60, 9), (10, 3)], "bf16", 64, seed=10)
    c.prefix[0] = 74  # slots 6 .. 8 would be at 80 .. 82 of 80
    c.table = np.ascontiguousarray(c.table[:, :5])
    c.to_gpu().call()
    c.check("beyond")
    c.prefix[1] = 1 << 30
    c.to_gpu().call()
    c.check("far beyond")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_what_a_slot_does_not_see_has_no_part(dtype, what):
    """Rows past the contexts, other branches of the tree and unused pages hold infinities or not-a-numbers."""
    val = float("nan") if what == "nan" else float("inf")
    c = Case([(50, 9), (21, 4), (96, 30), (70, 1)], dtype, 64, seed=11)
    seen = set()
    for b, (p, n) in enumerate(zip(c.prefix, np.diff(c.off))):
        seen |= {(int(c.table[b, x // 16]), x % 16) for x in range(p + n)}
    for page in range(c.pool.shape[1]):
        for row in range(16):
            if (page, row) not in seen:
                c.pool[:, page, 0, :, row * 64:(row + 1) * 64] = val
                c.pool[:, page, 1, :, row::16] = -val
    # slot 5 of user 0 and slot 17 of user 2: nobody is below them
    for b, j in ((0, 5), (2, 17)):
        s = c.off[b]
        c.parent[s:c.off[b + 1]][c.parent[s:c.off[b + 1]] == j] = 0
        x = int(c.prefix[b]) + j
        page, row = int(c.table[b, x // 16]), x % 16
        c.pool[:, page, 1, 0, row::16] = val
        c.pool[:, page, 1, 1, 5 * 16 + row] = -val
        c.pool[:, page, 0, 1, row * 64 + 3] = float("nan")
    c.to_gpu().call()
    c.check(f"{dtype} {what}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_seen_pass_on_their_infinities(dtype):
    c = Case([(50, 9), (21, 4)], dtype, 64, kind="chain", seed=12)
    for b, j, d, val in ((0, 3, 7, float("inf")), (0, 5, 7, float("-inf")), (0, 4, 9, float("-inf")), (1, 2, 1, float("nan"))):
        x = int(c.prefix[b]) + j
        c.pool[:, int(c.table[b, x // 16]), 1, :, d * 16 + x % 16] = val
    x = 13  # a cached token that every slot of user 1 sees
    c.pool[:, int(c.table[1, 0]), 1, 1, 20 * 16 + x] = float("inf")
    c.to_gpu().call()
    c.check(f"{dtype} seen")


@pytest.mark.parametrize("dtype,G,planes", [("bf16", 4, 1), ("bf16", 40, 2), ("f32", 4, 1)])
def test_scores_of_minus_infinity_weigh_nothing(dtype, G, planes):
    """Whole blocks whose scores are minus infinity or hugely negative, before and between others.  Their weights are
    0 exactly, so what the other keys' scores allow is the tolerance."""
    for val in (float("-inf"), -(2.0 ** 100)):
        c = Case([(1300, 9), (40, 3)], dtype, 64, 1, G, planes=planes, seed=21)
        c.q[:, :, 3] = 1.0
        if planes == 2:
            c.q_lo[:, :, 3] = 2.0 ** -10
        plain = c.pool.clone()
        for x in [*range(0, 600), *range(640, 900), 1301]:
            at = int(c.table[0, x // 16]), 0, slice(None), (x % 16) * 64 + 3
            c.pool[:, at[0], at[1], at[2], at[3]] = val
            plain[:, at[0], at[1], at[2], at[3]] = 0
        c.to_gpu().call()
        c.check(f"{dtype} {val}", scores_of=plain)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
def test_huge_scores_pick_the_largest(dtype, sign):
    """Scores of +-2^60 (1 + i): all weight on one token, whose value is the output."""
    c = Case([(70, 5), (16, 1)], dtype, 64, 1, 4, kind="chain", seed=22)
    c.q[:] = 0
    c.q[:, :, 3] = 1.5  # (so that a score times the scale is rounded)
    for b in range(2):
        for x in range(int(c.prefix[b]) + int(np.diff(c.off)[b])):
            c.pool[:, int(c.table[b, x // 16]), 0, :, (x % 16) * 64 + 3] = sign * 2.0 ** 60 * (1 + x % 61)
    c.to_gpu().call(scale=0.7)
    got = c.out.cpu().reshape(c.T, c.hq, 64)
    for b in range(2):
        for j in range(int(np.diff(c.off)[b])):
            keys = [x % 61 for x in range(int(c.prefix[b]) + j + 1)]
            x = [i for i, k in enumerate(keys) if k == (max(keys) if sign > 0 else min(keys))]
            pages = [c.pool[c.layer, int(c.table[b, i // 16]), 1, 0, i % 16::16] for i in x]
            want = torch.stack(pages).double().mean(0)
            assert len(x) <= 2
            err = (got[int(c.off[b]) + j].double() - want).abs().max().item()
            # (two equal weights: half of a sum of two bf16 values, rounded once to the output's type)
            assert err <= want.abs().max().item() * 2.0 ** (-8 if dtype == "bf16" else -22), (b, j, err)


def test_large_and_equal_scores():
    c = Case([(200, 8), (0, 5)], "bf16", 64, seed=13)
    c.q *= 30
    c.pool[:, :, 0] *= 4
    c.to_gpu().call()
    c.check("large scores")
    c = Case([(200, 8), (0, 5)], "bf16", 64, seed=14)
    c.pool[:, :, 0] = 0.5
    c.to_gpu().call()
    c.check("equal scores")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_pool_beyond_32_bits(dtype):
    """Pages whose elements are counted beyond 32 bits in the second of two layers."""
    c = Case([(300, 9), (17, 4), (64, 1)], dtype, 128, 8, 2, seed=23).to_gpu()
    pages, n = 70000, c.pool.shape[1]
    at = np.concatenate([[0, 3], np.linspace(30000, pages - 1, n - 2).astype(int)])
    big = torch.empty(2 * pages * 2 * 8 * 16 * 128, dtype=DT[dtype], device="cuda")
    assert big.numel() > 1 << 32
    big.view(2, pages, 2, 8, 16 * 128)[:, torch.from_numpy(at).cuda()] = c.d_pool
    c.kv = sv.make_kv_pool(big, 2, pages, 8, 128)
    c.d[2].copy_(torch.from_numpy(np.where(c.table >= 0, at[c.table], -1).astype(np.int32)))
    c.call()
    c.check(f"{dtype} beyond 32 bits")


def test_runs_are_equal_and_do_not_depend_on_the_workspace():
    c = Case([(900, 13), (40, 2), (300, 30)], "bf16", 128, 2, 8, planes=2, seed=15).to_gpu()
    c.call()
    first = c.out.clone(), c.out_lo.clone()
    c.ws.fill_(255)
    c.call()
    assert torch.equal(first[0], c.out) and torch.equal(first[1], c.out_lo)


def test_captured_calls_follow_their_arrays():
    """A graph replays with other trees, contexts, pages and queries; eager work of the
    program lies between the replays, and every replay equals the eager call."""
    c = Case([(700, 9), (30, 3), (0, 1), (100, 16)], "bf16", 128, 2, 4, planes=2, seed=16).to_gpu()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    c.call(stream=st)
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        c.call(stream=st)
    r = np.random.default_rng(17)
    for k in range(5):
        c.prefix = np.array([r.integers(0, 701), r.integers(0, 31), 0, r.integers(0, 101)], np.int32)
        cuts = np.sort(r.integers(0, c.T + 1, 3))
        c.off = np.minimum(np.concatenate([[0], cuts, [c.T]]), c.T).astype(np.int32)
        for b in range(4):  # contexts that the users' pages hold
            room = 16 * len(set(c.table[b])) if b != 2 else 16
            c.prefix[b] = min(c.prefix[b], max(0, room - 16))
        c.parent = r.integers(-1, 8, c.T).astype(np.int32)
        q = torch.randn(c.q.shape, generator=torch.Generator().manual_seed(k))
        c.q = q.to(torch.bfloat16)
        c.q_lo = (q - c.q.float()).to(torch.bfloat16)
        for dst, src in zip(c.d, (c.off, c.prefix, c.table, c.parent)):
            dst.copy_(torch.from_numpy(np.ascontiguousarray(src)))
        c.d_q.copy_(c.q)
        c.d_lo.copy_(c.q_lo)
        c.out.fill_(-7.0)
        c.out_lo.fill_(-7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = c.out.clone(), c.out_lo.clone()
        c.out.fill_(-7.0)
        c.out_lo.fill_(-7.0)
        c.ws.fill_(k)
        c.call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], c.out) and torch.equal(got[1], c.out_lo), k
    c.check("last replay")


def test_two_streams_at_once():
    cs = [Case([(1200, 9), (30, 30)], "bf16", 128, 2, 4, seed=18 + i).to_gpu() for i in range(2)]
    for c in cs:
        c.call()
    torch.cuda.synchronize()
    want = [c.out.clone() for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(20):
        for c, s in zip(cs, streams):
            c.call(stream=s)
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        assert torch.equal(c.out, w)


def test_binding_refuses_what_does_not_fit():
    c = Case([(20, 3), (4, 2)], "bf16", 64, seed=20).to_gpu()
    with pytest.raises(ValueError):
        sv.make_kv_pool(c.d_pool, 2, c.pool.shape[1] + 1, 2, 64)
    with pytest.raises(ValueError):
        sv.make_tree(c.d[0], c.d[1][:1], c.d[2], c.d[3], max_slots=3)
    with pytest.raises(ValueError):
        sv.make_tree(c.d[0], c.d[1], c.d[2], max_slots=3)
    with pytest.raises(ValueError):
        sv.make_tree(c.d[0], c.d[1], c.d[2].t(), c.d[3], max_slots=3)
    bad = [dict(q=c.d_q[:4]), dict(q=c.d_q.float()), dict(out=c.out[:4]), dict(out=c.out.transpose(0, 1)),
           dict(q=c.d_q.cpu()), dict(q_lo=c.d_q[:, :, ::2]), dict(ws=c.ws.cpu())]
    for b in bad:
        k = dict(q=c.d_q, out=c.out, q_lo=None, ws=c.ws)
        k.update(b)
        with pytest.raises(ValueError):
            sv.sd_tree_attention(c.kv, 0, c.tree, k["q"], k["out"], k["ws"], q_lo=k["q_lo"])
    with pytest.raises(sv.SdError) as e:
        sv.sd_tree_attention(c.kv, 2, c.tree, c.d_q, c.out, c.ws)
    assert e.value.status == sv.SD_EINVAL
    with pytest.raises(sv.SdError) as e:
        sv.sd_tree_attention(c.kv, 0, c.tree, c.d_q, c.out, c.ws[:0])
    assert e.value.status in (sv.SD_EINVAL, sv.SD_ENOMEM)
