"""Pins of the oracle's definitions of trees of drafts (oracle.trees): torch's
attention under an explicit mask, chains against the causal form, hand-worked
walks, moves and rows of logits."""
import numpy as np
import pytest
import torch

from oracle import trees


def random_parents(r, n):
    return np.array([-1] + [int(r.integers(0, j)) for j in range(1, n)], np.int64)[:n]


def test_paths():
    par = [-1, 0, 0, 1, 3, 2, 9]
    assert [trees.path_to(par, j) for j in range(7)] == [[0], [1, 0], [2, 0], [3, 1, 0], [4, 3, 1, 0], [5, 2, 0], [6]]


@pytest.mark.parametrize("seed", range(6))
def test_attention_is_torchs_under_the_tree_mask(seed):
    r = np.random.default_rng(seed)
    hkv, G, hd, pages = 2, 3, 8, 9
    prefix, n = int(r.integers(0, 70)), int(r.integers(1, 12))
    pool = r.standard_normal((2, pages, 2, hkv, 16 * hd))
    table = r.permutation(pages)[:6].reshape(1, 6)
    par = random_parents(r, n)
    q = r.standard_normal((n, hkv * G, hd))
    out, _, _ = trees.tree_attention(pool, 1, [0, n], [prefix], table, par, q, 0.3, hkv, 16)
    ctx = prefix + n
    mask = torch.zeros((n, ctx), dtype=torch.bool)
    mask[:, :prefix] = True
    for j in range(n):
        a = j
        while a >= 0:
            mask[j, prefix + a] = True
            a = int(par[a])
    for h in range(hkv * G):
        k = np.stack([pool[1, table[0, p // 16], 0, h // G].reshape(16, hd)[p % 16] for p in range(ctx)])
        v = np.stack([pool[1, table[0, p // 16], 1, h // G].reshape(hd, 16)[:, p % 16] for p in range(ctx)])
        ref = torch.nn.functional.scaled_dot_product_attention(
            torch.tensor(q[None, :, h]), torch.tensor(k[None]), torch.tensor(v[None]), attn_mask=mask[None], scale=0.3)
        assert np.abs(out[:, h] - ref[0].numpy()).max() < 1e-12


def test_no_parents_is_a_chain_and_pages_outside_do_not_count():
    r = np.random.default_rng(3)
    pool = r.standard_normal((1, 4, 2, 1, 16 * 4))
    q = r.standard_normal((5, 1, 4))
    table = np.array([[2, 0, 3]])
    a = trees.tree_attention(pool, 0, [0, 5], [30], table, None, q, 1.0, 1, 8)[0]
    b = trees.tree_attention(pool, 0, [0, 5], [30], table, [-1, 0, 1, 2, 3], q, 1.0, 1, 8)[0]
    assert np.array_equal(a, b)
    # without its second page a slot sees the first 16 tokens and, from position 32 on, its own page
    c = trees.tree_attention(pool, 0, [0, 5], [30], np.array([[2, 7, 3]]), None, q, 1.0, 1, 8)[0]
    d = trees.tree_attention(pool, 0, [0, 2], [16], np.array([[2]]), None, q[:2], 1.0, 1, 8)[0]
    assert np.allclose(c[:2], d, atol=1e-14)
    # nothing to see
    z = trees.tree_attention(pool, 0, [0, 1], [0], np.array([[-1]]), None, q[:1], 1.0, 1, 8)[0]
    assert (z == 0).all()


def test_slots_of_nobody():
    slots = trees.users_of([2, 4, 3, 9], [1, -5, 7], 6, 2)
    assert slots == [(2, 2, 1), (4, 0, 0), (3, 2, 7)]


def test_moves():
    pool = np.arange(1 * 3 * 2 * 1 * 32, dtype=np.float64).reshape(1, 3, 2, 1, 32)  # head_dim 2
    out = trees.copy_pages(pool, [0, 5, 1], [2, 1, -1])
    assert np.array_equal(out[0, 2], pool[0, 0]) and np.array_equal(out[0, :2], pool[0, :2])
    table = np.array([[1, 0]])
    out = trees.compact(pool, [14], table, np.array([[0, 3, 1, 9, 60]]), [5], 2)
    k = lambda p, i: p[0, i // 16, 0, 0].reshape(16, 2)[i % 16]  # noqa: E731
    v = lambda p, i: p[0, i // 16, 1, 0].reshape(2, 16)[:, i % 16]  # noqa: E731
    at = lambda pos: 16 * table[0, pos // 16] + pos % 16  # noqa: E731
    for i, src in enumerate([0, 3, 1, 9]):
        assert np.array_equal(k(out, at(14 + i)), k(pool, at(14 + src)))
        assert np.array_equal(v(out, at(14 + i)), v(pool, at(14 + src)))
    changed = {at(14 + i) for i in (1, 2, 3)}
    for i in range(48):
        if i not in changed:
            assert np.array_equal(k(out, i), k(pool, i)) and np.array_equal(v(out, i), v(pool, i))


def test_walks():
    drafts, parent = [7, 8, 7, 9, 8, 7], [0, 0, 1, 1, 2, 0]
    assert trees.walk([7, 9, 0, 0, 3, 0, 0], drafts, parent) == ([1, 4], 3)
    assert trees.walk([8, 0, 8, 0, 0, 11, 0], drafts, parent) == ([2, 5], 11)
    assert trees.walk([5] * 7, drafts, parent) == ([], 5)
    assert trees.walk([7, 5, 5, 5, 5, 5, 4], drafts, parent) == ([1], 5)  # the first of equal drafts
    assert trees.walk([-1] * 7, drafts, parent) == ([], -1)


def test_rows_of_logits():
    z = [2.0, -2.0, 1.0, 0.0, 4.0, -np.inf]
    out = trees.adjust_row(z, prompt=[0, 1, 99, -1], output=[1, 1, 2, 5], repetition=2.0, presence=0.5, frequency=0.25,
                           biases=[(3, 1.0), (4, 5.0), (4, -1.0), (77, 3.0)], allowed=[1, 1, 1, 1, 1, 1])
    assert out.tolist() == [1.0, -4.0 - 1.0, 0.5 - 0.75, 1.0, 3.0, -np.inf]
    out = trees.adjust_row(z, output=[0], repetition=-1.0, presence=np.nan, frequency=np.inf, allowed=[1, 0, 1, 1, 0, 1])
    assert out.tolist() == [2.0, -np.inf, 1.0, 0.0, -np.inf, -np.inf]
