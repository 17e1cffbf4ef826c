"""Forks on a busy stream (sd_user_fork): their pages may be given back, handed out and
written on other streams at once, and the copies read and write what they were
meant to."""
import numpy as np
import pytest
import torch

import workload as wl
from gpu_harness import load_synthetic_kv, make_verifier
from paper_2604_20919_amd import sdverify as sv
from workload.device import DeviceWeights

pytestmark = pytest.mark.gpu

N = 200  # cached tokens of the source


class Forks:
    """User 0 with a cache; a stream that is busy for some tens of milliseconds, and another."""

    def __init__(self, users=4):
        self.w = wl.custom_workload("tiny-bf16", [N] + [0] * (users - 1), [3] * users, seed=91)
        self.m = self.w.model
        self.dw = DeviceWeights(self.m, self.w.seed)
        self.v = make_verifier(self.w, self.dw, extra_ctx=2 * N)
        load_synthetic_kv(self.v, self.w, users=[0])
        self.v.reset_user(0, N, 5)
        self.want = self.rows(0, N)
        self.busy, self.other = torch.cuda.Stream(), torch.cuda.Stream()
        self.a = torch.randn((8192, 8192), dtype=torch.bfloat16, device="cuda")
        self.out = torch.empty_like(self.a)
        torch.mm(self.a, self.a, out=self.out)
        torch.cuda.synchronize()

    def work(self):
        with torch.cuda.stream(self.busy):
            for _ in range(40):  # about a millisecond each
                torch.mm(self.a, self.a, out=self.out)
            self.worked = torch.cuda.Event()
            self.worked.record()

    def rows(self, u, n):
        """Keys and values of a user in all layers."""
        got = []
        for l in range(self.m.n_layers):
            k = torch.empty((n, self.m.n_kv_heads, self.m.head_dim), dtype=torch.int16, device="cuda")
            x = torch.empty_like(k)
            self.v.read_kv(u, l, 0, k, x)
            got += [k, x]
        torch.cuda.synchronize()
        return torch.stack(got).cpu()

    def full(self, n, value):
        x = torch.full((n, self.m.n_kv_heads, self.m.head_dim), value, dtype=torch.int16, device="cuda")
        torch.cuda.synchronize()
        return x

    def write(self, u, x, stream):
        """Makes a user's rows x, in all layers."""
        for l in range(self.m.n_layers):
            self.v.write_kv(u, l, 0, x, x, stream)
        print("written while the copy waits:", not self.worked.query(), flush=True)


def test_a_source_released_and_its_pages_written_elsewhere():
    f = Forks()
    held = set(f.v.user_pages(0))
    x = f.full(N, 77)
    f.work()
    f.v.fork_user(1, 0, N, 5, stream=f.busy)
    sv.sd_user_release(f.v.ctx, 0)
    f.v.reset_user(2, N, 1)
    assert held & set(f.v.user_pages(2))
    f.write(2, x, f.other)
    torch.cuda.synchronize()
    assert torch.equal(f.rows(1, N), f.want)
    assert (f.rows(2, N) == 77).all()
    f.v.close()


def test_a_source_shortened():
    f = Forks()
    held = set(f.v.user_pages(0)[1:])
    x = f.full(N - 20, 78)
    f.work()
    f.v.fork_user(1, 0, N, 5, stream=f.busy)
    f.v.reset_user(0, 3, 1)
    f.v.reset_user(2, N - 20, 1)
    assert held >= set(f.v.user_pages(2))
    f.write(2, x, f.other)
    torch.cuda.synchronize()
    assert torch.equal(f.rows(1, N), f.want)
    assert (f.rows(2, N - 20) == 78).all()
    f.v.close()


@pytest.mark.parametrize("again", ["released", "forked shorter"])
def test_a_target_given_back_before_its_copy_has_run(again):
    """The copy must not land on what its pages' next owner wrote."""
    f = Forks()
    x = f.full(N - 20, 79)
    f.work()
    f.v.fork_user(1, 0, N, 5, stream=f.busy)
    held = set(f.v.user_pages(1))
    if again == "released":
        sv.sd_user_release(f.v.ctx, 1)
    else:
        f.v.fork_user(1, 0, 10, 6, stream=f.other)
    f.v.reset_user(2, N - 20, 1)
    assert held >= set(f.v.user_pages(2))
    f.write(2, x, f.other)
    torch.cuda.synchronize()
    assert (f.rows(2, N - 20) == 79).all()
    assert torch.equal(f.rows(0, N), f.want)
    if again != "released":
        assert torch.equal(f.rows(1, 10), f.want[:, :10])
    f.v.close()


def test_forks_of_one_source_and_of_forks_on_many_streams():
    """Copies of a page follow each other, whichever streams they are on."""
    f = Forks(users=6)
    streams = [f.busy, f.other] + [torch.cuda.Stream() for _ in range(2)]
    x = f.full(N, 80)
    f.work()
    f.v.fork_user(1, 0, N, 5, stream=streams[0])
    f.v.fork_user(2, 1, N, 5, stream=streams[1])       # of a copy that has not run
    f.v.fork_user(3, 0, N - 9, 5, stream=streams[2])
    f.v.fork_user(4, 3, 50, 5, stream=streams[3])
    sv.sd_user_release(f.v.ctx, 0)
    sv.sd_user_release(f.v.ctx, 1)
    f.v.fork_user(5, 2, N, 5, stream=streams[3])
    f.v.reset_user(0, N, 1)
    f.write(0, x, streams[2])
    torch.cuda.synchronize()
    for u, n in ((2, N), (3, N - 9), (4, 50), (5, N)):
        assert torch.equal(f.rows(u, n), f.want[:, :n]), u
    assert (f.rows(0, N) == 80).all()
    f.v.close()


@pytest.mark.parametrize("graph", [False, True])
def test_passes_come_after_the_copies_of_their_pages(graph):
    """A pass of the fork on another stream, and one of a user with the source's former pages."""
    f = Forks()
    d = torch.zeros(6, dtype=torch.int32, device="cuda")
    L = np.array([3] * 4, np.int32)

    def run(users):
        assign = np.array([0 if u in users else -1 for u in range(4)], np.int32)
        if graph:
            f.v.verify(0, assign, L, d, None, "greedy", stream=f.other, graph=True)
        else:
            f.v.verify(0, assign, L, d, None, "greedy", stream=f.other)
        lg = f.v.logits(0, 4 * len(users), f.other)
        f.v.accept(0, 4)
        return lg.cpu().numpy()

    torch.cuda.synchronize()
    want = run([0])
    f.work()
    f.v.fork_user(1, 0, N, 5, stream=f.busy)
    assert np.array_equal(run([1]), want)  # (a user of its own in the batch, the same sums)
    sv.sd_user_release(f.v.ctx, 1)
    f.work()
    f.v.fork_user(1, 0, N, 5, stream=f.busy)
    sv.sd_user_release(f.v.ctx, 0)
    f.v.reset_user(2, 0, 5)
    run([2])  # writes its rows into a page of the source
    torch.cuda.synchronize()
    assert torch.equal(f.rows(1, N), f.want)
    f.v.close()


def test_many_forks_one_after_the_other():
    """Events come back: forks, releases and writes in turn on two streams."""
    f = Forks()
    for i in range(200):
        s = (f.busy, f.other)[i % 2]
        f.v.fork_user(1 + i % 2, 0, N - i % 50, 5, stream=s)
        f.v.fork_user(2 - i % 2, 1 + i % 2, 40, 5, stream=(f.other, f.busy)[i % 2])
    torch.cuda.synchronize()
    assert torch.equal(f.rows(2, N - 49), f.want[:, :N - 49]) and torch.equal(f.rows(1, 40), f.want[:, :40])
    f.v.close()


def test_forks_and_writes_under_capture():
    """A captured fork and write run with their graph, another stream's fork at once."""
    f = Forks()
    f.v.reset_user(3, N, 1)
    x = torch.full((N, f.m.n_kv_heads, f.m.head_dim), 81, dtype=torch.int16, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=f.other):
        f.v.fork_user(1, 0, N, 5, stream=f.busy)  # (not captured)
        f.v.fork_user(2, 0, N, 5, stream=f.other)
        f.v.write_kv(3, 0, 0, x, x, f.other)
    torch.cuda.synchronize()
    for _ in range(3):
        f.v.write_kv(2, 0, 0, x, x)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(f.rows(2, N), f.want) and torch.equal(f.rows(1, N), f.want)
        assert (f.rows(3, N)[:2] == 81).all()
    f.v.close()
