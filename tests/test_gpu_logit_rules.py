"""Rules on logits (sd_adjust_logits) against their 64-bit definition (oracle.trees).

Tolerance: the division or product, the product and sum of the penalties, the
subtraction and the bias round once each in fp32, by 2^-24 of what they have in
hand: at most 5 * 2^-24 * (|z| max(r, 1/r) + |f| c + |p| + |bias|) with the last
rounding.  What no rule touches is equal."""
import numpy as np
import pytest
import torch

from oracle import trees
from paper_2604_20919_amd import sdverify as sv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


class Rules:
    """Random rules of n rows over V tokens: `users` histories, each for some rows in a row."""

    def __init__(self, n, V, seed, users=3, hist=50, biases=5, masks=True, drafts=True, penalties=True, odd=False):
        r = np.random.default_rng(seed)
        self.n, self.V = n, V
        first = np.sort(r.choice(np.arange(1, n), min(users, n) - 1, replace=False)) if n > 1 and users > 1 else np.array([], int)
        start = np.concatenate([[0], first, [n]])
        self.user = np.repeat(np.arange(start.size - 1), np.diff(start))
        U = start.size - 1
        size = r.integers(0, hist + 1, U)
        at = np.concatenate([[0], np.cumsum(size)])
        wide = max(1, V // 3)
        self.tokens = r.integers(0, wide, at[-1]) * (1 if not odd else r.choice([1, -1, 5], at[-1]))
        self.hist = np.array([[at[u], at[u] + r.integers(0, size[u] + 1) if size[u] else at[u], at[u + 1]] for u in range(U)])[self.user]
        self.rep = r.choice([1.0, 1.3, 0.8], n).astype(np.float32)
        self.pres = r.choice([0.0, 0.7, -0.4], n).astype(np.float32)
        self.freq = r.choice([0.0, 0.3, -0.2], n).astype(np.float32)
        self.row_token = r.integers(0, wide, n)
        self.row_parent = np.array([r.integers(start[self.user[t]], t) if t > start[self.user[t]] else -1 for t in range(n)])
        m = r.integers(0, biases + 1, U) if biases else np.zeros(U, int)
        ba = np.concatenate([[0], np.cumsum(m)])
        self.bias_token = r.integers(0, wide, ba[-1])  # some twice
        self.bias_value = r.standard_normal(ba[-1]).astype(np.float32) * 3
        self.bias = np.array([[ba[u], ba[u + 1]] for u in range(U)])[self.user]
        self.words = r.integers(-2 ** 31, 2 ** 31, (4, (V + 31) // 32)).astype(np.int32)
        self.words[3] = 0  # allows nothing
        self.mask_row = r.choice([-1, 0, 1, 2, 3, 4, 99], n)
        self.use = dict(hist=hist > 0, drafts=drafts, biases=biases > 0, masks=masks, penalties=penalties)
        if odd:
            self.rep = r.choice(np.array([-1.0, 0.0, np.nan, np.inf, 1.5], np.float32), n)
            self.pres = r.choice(np.array([np.nan, np.inf, -np.inf, 0.5], np.float32), n)
            self.freq = r.choice(np.array([np.nan, np.inf, 0.25], np.float32), n)
            self.hist = self.hist + r.integers(-8, 9, self.hist.shape)
            self.bias = self.bias + r.integers(-4, 5, self.bias.shape)
            self.row_parent = r.integers(-3, n + 3, n)
            self.row_token = self.row_token * r.choice([1, -1, 7], n)

    def make(self):
        u, k = self.use, {}
        if u["hist"]:
            k.update(tokens=dev(self.tokens, np.int32), hist=dev(self.hist, np.int32))
        if u["penalties"]:
            k.update(repetition=dev(self.rep, np.float32), presence=dev(self.pres, np.float32), frequency=dev(self.freq, np.float32))
        if u["drafts"]:
            k.update(row_token=dev(self.row_token, np.int32), row_parent=dev(self.row_parent, np.int32))
        if u["biases"]:
            k.update(bias_token=dev(self.bias_token, np.int32), bias_value=dev(self.bias_value, np.float32),
                     bias=dev(self.bias, np.int32))
        if u["masks"]:
            k.update(mask=dev(self.words, np.int32), mask_row=dev(self.mask_row, np.int32))
        return sv.make_logit_rules(self.n, self.V, **k)

    def ranges(self, t):
        N, M = self.tokens.size, self.bias_token.size
        b = min(max(int(self.hist[t, 0]), 0), N)
        f = min(max(int(self.hist[t, 1]), b), N)
        e = min(max(int(self.hist[t, 2]), f), N)
        ob = min(max(int(self.bias[t, 0]), 0), M)
        return b, f, e, ob, min(max(int(self.bias[t, 1]), ob), M)

    def row(self, t, z):
        """(row, tolerance) in 64 bits."""
        u = self.use
        b, f, e, ob, oe = self.ranges(t)
        prompt, output = (list(self.tokens[b:f]), list(self.tokens[f:e])) if u["hist"] else ([], [])
        if u["drafts"]:
            output += [self.row_token[a] for a in trees.path_to(self.row_parent, t) if a >= t - 256]
        biases = list(zip(self.bias_token[ob:oe], self.bias_value[ob:oe])) if u["biases"] else []
        allowed = None
        if u["masks"] and 0 <= self.mask_row[t] < 4:
            allowed = np.unpackbits(self.words[self.mask_row[t]].view(np.uint8), bitorder="little")[:self.V] == 1
        opt = (self.rep[t], self.pres[t], self.freq[t]) if u["penalties"] else (1.0, 0.0, 0.0)
        want = trees.adjust_row(z, prompt, output, *opt, biases, allowed)
        rep = opt[0] if opt[0] > 0 and np.isfinite(opt[0]) else 1.0
        fin = [x if np.isfinite(x) else 0.0 for x in opt[1:]]
        with np.errstate(invalid="ignore", over="ignore"):
            tol = np.abs(z) * max(rep, 1 / rep)
        tol = np.where(np.isfinite(tol), tol, 0.0) + abs(fin[0]) + abs(fin[1]) * len(output) + max([abs(v) for _, v in biases] + [0.0])
        touched = np.zeros(self.V, bool)
        for x in prompt + output + [k for k, _ in biases]:
            if 0 <= x < self.V:
                touched[x] = True
        return want, np.where(touched, 5 * 2.0 ** -24 * tol, 0.0)


def logits(n, V, dtype, seed, kind="plain", pad=0):
    r = np.random.default_rng(seed + 77)
    z = (r.standard_normal((n, V)) * 3).astype(np.float32)
    if kind == "odd":
        z = np.where(r.random((n, V)) < 0.2, r.choice(np.array([np.inf, -np.inf, np.nan, 0.0, -0.0, 1e-40], np.float32), (n, V)), z)
    buf = torch.full((n, V + pad), 5.0, dtype=DT[dtype], device="cuda")
    buf[:, :V] = torch.from_numpy(z).cuda()
    return buf[:, :V]


def check(R, z, out, label):
    torch.cuda.synchronize()
    zz, got = z.double().cpu().numpy(), out.double().cpu().numpy()
    for t in range(R.n):
        want, tol = R.row(t, zz[t])
        nan = np.isnan(want)
        assert np.array_equal(np.isnan(got[t]), nan), f"{label}: not-a-numbers of row {t}"
        with np.errstate(invalid="ignore"):
            off = np.abs(got[t] - want)
        off = np.where(nan | (got[t] == want), 0.0, off)
        assert (off <= tol).all(), f"{label}: row {t} token {int(np.argmax(off - tol))} is {off.max()} off"


@pytest.mark.parametrize("n,V", [(1, 1), (1, 151936), (3, 31), (5, 4095), (2, 4096), (7, 4097), (40, 1000), (9, 32003), (300, 64),
                                 (1, 2), (65, 8192)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows(n, V, dtype):
    R = Rules(n, V, n + V, users=max(1, n // 4))
    z = logits(n, V, dtype, n)
    out = torch.empty((n, V), device="cuda")
    sv.sd_adjust_logits(z, R.make(), out)
    check(R, z, out, f"{n}x{V} {dtype}")


@pytest.mark.parametrize("off", [dict(hist=0), dict(drafts=False), dict(biases=0), dict(masks=False), dict(penalties=False),
                                 dict(hist=0, biases=0, masks=False), dict(hist=0, drafts=False, penalties=False, biases=0),
                                 dict(hist=0, drafts=False, penalties=False, masks=False)])
def test_each_rule_alone_and_left_out(off):
    R = Rules(11, 5000, 3, **off)
    z = logits(11, 5000, "f32", 3)
    out = torch.empty((11, 5000), device="cuda")
    sv.sd_adjust_logits(z, R.make(), out)
    check(R, z, out, str(off))


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_value_means_something(seed, dtype):
    """Options, ranges, tokens and parents out of range; infinities and not-a-numbers among the logits."""
    R = Rules(23, 4200 + seed, seed, users=5, hist=300, biases=40, odd=True)
    z = logits(23, 4200 + seed, dtype, seed, "odd", pad=seed)
    out = torch.empty((23, 4200 + seed), device="cuda")
    sv.sd_adjust_logits(z, R.make(), out)
    check(R, z, out, f"odd {seed}")


@pytest.mark.parametrize("V,pad,opad", [(4096, 4, 8), (4096, 1, 0), (4100, 0, 3), (151936, 24, 0), (1003, 5, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(V, pad, opad, dtype):
    R = Rules(6, V, V + pad)
    z = logits(6, V, dtype, pad, pad=pad)
    buf = torch.full((6, V + opad), 9.0, device="cuda")
    sv.sd_adjust_logits(z, R.make(), buf[:, :V])
    check(R, z, buf[:, :V], f"{V}+{pad} {dtype}")
    assert (buf[:, V:] == 9.0).all()


@pytest.mark.parametrize("V,pad", [(4096, 0), (5001, 0), (5000, 8), (300, 1)])
def test_in_place(V, pad):
    R = Rules(17, V, 9)
    z = logits(17, V, "f32", 9, "odd", pad)
    before = z.clone()
    sv.sd_adjust_logits(z, R.make(), z)
    check(R, before, z, f"in place {V}")


@pytest.mark.parametrize("n,V,users", [(1, 3000, 1), (17, 9001, 5), (40, 6000, 13)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_biases(n, V, users, dtype):
    """More biases than a workgroup has threads, many of one token, next to users of few."""
    R = Rules(n, V, n, users=users, hist=7000, biases=3500)
    z = logits(n, V, dtype, n)
    out = torch.empty((n, V), device="cuda")
    sv.sd_adjust_logits(z, R.make(), out)
    check(R, z, out, f"{n}x{V} {dtype}")


def test_rows_far_apart():
    """Rows of logits and results whose elements are counted beyond 32 bits."""
    R = Rules(5, 700, 3)
    z = logits(5, 700, "f32", 3)
    step = (1 << 30) + 4
    far = torch.empty(4 * step + 700, device="cuda").as_strided((5, 700), (step, 1))
    far.copy_(z)
    out = torch.empty(4 * step + 704, device="cuda").as_strided((5, 700), (step + 1, 1))
    sv.sd_adjust_logits(far, R.make(), out)
    check(R, z, out, "apart")
    sv.sd_adjust_logits(far, R.make(), far)
    check(R, z, far, "in place")


def test_long_histories_and_deep_paths():
    R = Rules(260, 2000, 4, users=1, hist=20000, biases=300)
    R.row_parent = np.arange(-1, 259)  # a chain of 260: the first rows are too far below the last
    z = logits(260, 2000, "f32", 4)
    out = torch.empty((260, 2000), device="cuda")
    sv.sd_adjust_logits(z, R.make(), out)
    check(R, z, out, "long")


def test_many_rows():
    R = Rules(5000, 96, 5, users=900, hist=9)
    z = logits(5000, 96, "bf16", 5)
    out = torch.empty((5000, 96), device="cuda")
    sv.sd_adjust_logits(z, R.make(), out)
    check(R, z, out, "5000 rows")


def test_empty_lists():
    n, V = 3, 100
    z = logits(n, V, "f32", 6)
    out = torch.empty((n, V), device="cuda")
    none, rows = torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros((n, 3), dtype=torch.int32, device="cuda")
    r = sv.make_logit_rules(n, V, tokens=none, hist=rows, bias_token=none, bias_value=none.float(), bias=rows[:, :2].contiguous(),
                            mask=torch.empty((0, 4), dtype=torch.int32, device="cuda"), mask_row=rows[:, 0].contiguous())
    sv.sd_adjust_logits(z, r, out)
    torch.cuda.synchronize()
    assert torch.equal(out, z)


def test_a_masked_out_row_gives_no_token():
    """The rules, then the sampler: a row that allows nothing gives token -1, the others an allowed one."""
    n, V = 6, 5000
    R = Rules(n, V, 8, biases=0)
    R.mask_row = np.array([0, 3, 1, 3, -1, 2])
    z = logits(n, V, "bf16", 8)
    out = torch.empty((n, V), device="cuda")
    sv.sd_adjust_logits(z, R.make(), out)
    tok = torch.empty(n, dtype=torch.int32, device="cuda")
    ws = torch.empty(sv.sd_filter_query_size(n, V), dtype=torch.uint8, device="cuda")
    sv.sd_sample_filtered(out, torch.full((n,), 0.4, device="cuda"), tok, ws)
    torch.cuda.synchronize()
    tok = tok.cpu().numpy()
    assert (tok[[1, 3]] == -1).all()
    for t in (0, 2, 5):
        assert (int(R.words[R.mask_row[t], tok[t] // 32]) >> (tok[t] % 32)) & 1


def test_captured_rules_follow_their_arrays():
    R = Rules(30, 6000, 12, users=4)
    z = logits(30, 6000, "f32", 12)
    out = torch.empty((30, 6000), device="cuda")
    rules = R.make()
    st = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        sv.sd_adjust_logits(z, rules, out, stream=st)
    for k in range(4):
        S = Rules(30, 6000, 12, users=4)
        r = np.random.default_rng(k)
        S.row_token = r.integers(0, 2000, 30)
        S.rep = r.choice([1.0, 2.0], 30).astype(np.float32)
        S.mask_row = r.integers(-1, 4, 30)
        names = {2: S.rep, 5: S.row_token, 11: S.mask_row}
        for i, a in names.items():
            rules.tensors[i].copy_(torch.from_numpy(np.ascontiguousarray(a)))
        z.copy_(logits(30, 6000, "f32", 100 + k))
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        check(S, z, out, f"replay {k}")


def test_binding_refuses_what_does_not_fit():
    R = Rules(4, 100, 1)
    rules = R.make()
    z = logits(4, 100, "f32", 1)
    for zz, o in ((z[:3], z), (z, z[:3]), (z[:, :99], z), (z, z.bfloat16()), (z.cpu(), z), (z.double(), z)):
        with pytest.raises(ValueError):
            sv.sd_adjust_logits(zz, rules, o)
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    for k in (dict(), dict(tokens=i(5)), dict(tokens=i(5), hist=i(4, 2)), dict(tokens=i(5), hist=i(3, 3)), dict(row_token=i(4)),
              dict(mask=i(2, 3), mask_row=i(4)), dict(mask=i(2, 4), mask_row=i(5)), dict(bias_token=i(5), bias=i(4, 2)),
              dict(repetition=i(4)), dict(presence=torch.zeros(5, device="cuda"))):
        with pytest.raises(ValueError):
            sv.make_logit_rules(4, 100, **k)
