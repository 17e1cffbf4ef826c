"""Pages of a cache copied and rows moved together (sd_kv_copy_pages, sd_kv_compact)
against their definition (oracle.trees): bit for bit."""
import numpy as np
import pytest
import torch

from oracle import trees
from paper_2604_20919_amd import sdverify as sv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(dtype, layers, pages, hkv, hd, seed):
    g = torch.Generator().manual_seed(seed)
    host = torch.randn((layers, pages, 2, hkv, 16 * hd), generator=g).to(DT[dtype])
    dev = host.cuda()
    return host.double().numpy(), dev, sv.make_kv_pool(dev, layers, pages, hkv, hd)


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


@pytest.mark.parametrize("dtype,layers,pages,hkv,hd", [
    ("bf16", 1, 2, 1, 64), ("bf16", 3, 9, 2, 128), ("f32", 2, 5, 3, 64), ("f32", 2, 7, 1, 6), ("f32", 1, 4, 1, 2),
    ("bf16", 28, 40, 8, 128), ("f32", 2, 6, 5, 34)])
def test_pages(dtype, layers, pages, hkv, hd):
    host, dev, pool = make(dtype, layers, pages, hkv, hd, pages)
    order = np.random.default_rng(pages).permutation(pages)
    n = pages // 2
    src, dst = order[:n], order[n:2 * n]
    sv.sd_kv_copy_pages(pool, ints(src), ints(dst))
    torch.cuda.synchronize()
    assert np.array_equal(dev.double().cpu().numpy(), trees.copy_pages(host, src, dst))


def test_pages_outside_the_pool_copy_nothing():
    host, dev, pool = make("bf16", 2, 6, 2, 64, 1)
    src, dst = [0, -1, 6, 2, 1 << 30], [3, 4, 5, -7, 1]
    sv.sd_kv_copy_pages(pool, ints(src), ints(dst))
    torch.cuda.synchronize()
    assert np.array_equal(dev.double().cpu().numpy(), trees.copy_pages(host, src, dst))


def table_of(r, users, most, pages):
    return r.permutation(pages)[:users * most].reshape(users, most)


@pytest.mark.parametrize("dtype,layers,hkv,hd", [("bf16", 2, 2, 64), ("bf16", 3, 1, 128), ("f32", 2, 2, 64), ("f32", 1, 3, 10),
                                                 ("f32", 2, 1, 128), ("f32", 1, 1, 2)])
@pytest.mark.parametrize("kind", ["path", "any", "none", "odd"])
def test_rows(dtype, layers, hkv, hd, kind):
    r = np.random.default_rng(hd + layers)
    users, most, width = 7, 6, 12
    host, dev, pool = make(dtype, layers, users * most + 3, hkv, hd, hd)
    table = table_of(r, users, most, users * most + 3)
    prefix = np.array([0, 5, 15, 16, 17, 31, 60])
    n_keep = r.integers(0, width + 1, users)
    keep = np.full((users, width), -1)
    for b in range(users):
        if kind == "path":  # ascending, as accepted paths are; sources and destinations overlap
            keep[b] = np.sort(r.choice(30, width, replace=False))
        elif kind == "any":  # any order, some twice, some upwards
            keep[b] = r.integers(0, 30, width)
        elif kind == "odd":
            keep[b] = r.choice([-1, -9, 0, 3, 7, 31, 40, 1 << 30], width)
    if kind == "none":
        keep[:] = np.arange(width)
    if kind == "odd":
        n_keep[:3] = [99, -3, width]
        prefix[6] = -4
        table[4, 2], table[5, 3] = -1, users * most + 3
    sv.sd_kv_compact(pool, ints(prefix), ints(table), ints(keep), ints(n_keep))
    torch.cuda.synchronize()
    want = trees.compact(host, prefix, table, keep, n_keep, hd)
    assert np.array_equal(dev.double().cpu().numpy(), want), f"{dtype} {hd} {kind}"


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 128), ("f32", 50)])
def test_the_most_rows(dtype, hd):
    r = np.random.default_rng(5)
    host, dev, pool = make(dtype, 2, 40, 2, hd, 5)
    table = table_of(r, 1, 36, 40)
    keep = np.sort(r.choice(500, 256, replace=False)).reshape(1, 256)
    keep[0, 200:] = r.permutation(keep[0, 200:])
    for n in (256, 255, 1):
        sv.sd_kv_compact(pool, ints([37]), ints(table), ints(keep), ints([n]))
        torch.cuda.synchronize()
        host = trees.compact(host, [37], table, keep, [n], hd)
        assert np.array_equal(dev.double().cpu().numpy(), host), n


def test_a_pool_beyond_32_bits():
    """Pages whose elements are counted beyond 32 bits in the second of two layers."""
    r = np.random.default_rng(9)
    pages, page = 70000, 2 * 8 * 16 * 128
    big = torch.empty(2 * pages * page, dtype=torch.bfloat16, device="cuda")
    assert big.numel() > 1 << 32
    rows = big.view(2, pages, 2, 8, 16 * 128)
    at = np.array([0, 3, 34000, 51111, 65535, 65536, 69998, 69999])  # the small pool's pages in the large one
    host, dev, _ = make("bf16", 2, at.size, 8, 128, 9)
    where = torch.from_numpy(at).cuda()
    rows[:, where] = dev
    pool = sv.make_kv_pool(big, 2, pages, 8, 128)
    src, dst = [1, 6, 3], [7, 0, 4]
    sv.sd_kv_copy_pages(pool, ints(at[src]), ints(at[dst]))
    torch.cuda.synchronize()
    host = trees.copy_pages(host, src, dst)
    assert np.array_equal(rows[:, where].double().cpu().numpy(), host)
    table, prefix, keep, n_keep = r.permutation(at.size).reshape(2, 4), [11, 30], r.integers(0, 33, (2, 9)), [9, 7]
    sv.sd_kv_compact(pool, ints(prefix), ints(at[table]), ints(keep), ints(n_keep))
    torch.cuda.synchronize()
    assert np.array_equal(rows[:, where].double().cpu().numpy(), trees.compact(host, prefix, table, keep, n_keep, 128))


def test_bits_are_kept():
    """Not-a-numbers with payloads, infinities and subnormals move as they are."""
    r = np.random.default_rng(6)
    bits = torch.from_numpy(r.integers(-2 ** 15, 2 ** 15, (2, 8, 2, 2, 16 * 64)).astype(np.int16))
    dev = bits.cuda()
    pool = sv.make_kv_pool(dev.view(torch.bfloat16), 2, 8, 2, 64)
    sv.sd_kv_copy_pages(pool, ints([1, 2]), ints([5, 7]))
    sv.sd_kv_compact(pool, ints([9]), ints([[3, 0, 6]]), ints([[0, 4, 9, 30]]), ints([4]))
    torch.cuda.synchronize()
    want = trees.copy_pages(bits.numpy(), [1, 2], [5, 7])
    want = trees.compact(want, [9], np.array([[3, 0, 6]]), np.array([[0, 4, 9, 30]]), [4], 64)
    assert np.array_equal(dev.cpu().numpy(), want)


def test_captured_moves_follow_their_arrays():
    host, dev, pool = make("bf16", 2, 24, 2, 64, 7)
    r = np.random.default_rng(7)
    src, dst = ints([0, 1]), ints([22, 23])
    prefix, table, keep, n_keep = ints([3, 9]), ints(r.permutation(20)[:10].reshape(2, 5)), ints([[0, 2, 5], [0, 1, 7]]), ints([3, 3])

    def call(st):
        sv.sd_kv_copy_pages(pool, src, dst, stream=st)
        sv.sd_kv_compact(pool, prefix, table, keep, n_keep, stream=st)

    st = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        call(st)
    for k in range(4):
        a, b = r.integers(0, 20, 2), [22, 23]
        p, ke, n = r.integers(0, 40, 2), r.integers(0, 30, (2, 3)), r.integers(0, 4, 2)
        for t, v in ((src, a), (prefix, p), (keep, ke), (n_keep, n)):
            t.copy_(torch.from_numpy(np.ascontiguousarray(v, np.int32)))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        host = trees.compact(trees.copy_pages(host, a, b), p, table.cpu().numpy(), ke, n, 64)
        assert np.array_equal(dev.double().cpu().numpy(), host), k


def test_binding_refuses_what_does_not_fit():
    _, dev, pool = make("bf16", 2, 6, 2, 64, 8)
    one = ints([0])
    for f in (lambda: sv.sd_kv_copy_pages(pool, one, ints([0, 1])), lambda: sv.sd_kv_copy_pages(pool, one, one.long()),
              lambda: sv.sd_kv_copy_pages(pool, one.cpu(), one), lambda: sv.sd_kv_compact(pool, one, ints([[0], [1]]), ints([[0]]), one),
              lambda: sv.sd_kv_compact(pool, one, ints([[0]]), one, one)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(sv.SdError):
        sv.sd_kv_copy_pages(pool, one[:0], one[:0])
