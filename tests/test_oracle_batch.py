"""Pins of the batch oracle: closed forms, the other oracles and brute force."""
import numpy as np

from oracle import batch, rope
from tests.batch_util import ancestors, sections, theta, tree


def test_plan_by_hand():
    # pages of 4 tokens: request 0 holds 6 tokens in pages 9, 8 and gets 3 more; request 1 is empty and gets 1
    r = batch.plan(4, [6, 0], [3, 1], [2, 0], [[9, 8, -1], [-1, -1, -1]], [5, 7, 3], 1, 6)
    assert r["row_start"] == [0, 3, 4] and r["held"] == [3, 1] and r["head"] == 3
    assert r["table"] == [[9, 8, 7], [3, -1, -1]]
    assert r["slot"] == [8 * 4 + 2, 8 * 4 + 3, 7 * 4, 3 * 4, -1, -1]
    assert r["coords"] == [[6] * 3, [7] * 3, [8] * 3, [0] * 3] and r["mask"] == [1, 3, 7, 1]


def test_tree_masks_are_the_transitive_closure():
    rng = np.random.default_rng(0)
    n = 90
    par = tree(rng, n)
    a = np.eye(n, dtype=int)
    for i in range(n):
        if par[i] >= 0:
            a[i] |= a[par[i]]
    r = batch.plan(16, [5], [n], [1], [list(range(9))], list(range(20, 40)), 0, n, parent=par, base=[100])
    assert [[m >> w & 1 for w in range(n)] for m in r["mask"]] == a.tolist()
    assert [c[0] for c in r["coords"]] == (100 + a.sum(1) - 1).tolist()
    assert r["mask"] == ancestors(par)
    words = batch.mask_words(r["mask"], 2)
    assert [int(words[70, w // 64] >> (w % 64) & 1) for w in range(n)] == a[70].tolist()


def test_norm_and_rotation_against_the_rotation_oracle():
    rng = np.random.default_rng(1)
    x, d = rng.standard_normal((5, 3, 16)), 16
    co = rng.integers(0, 1000, (5, 3))
    sec = sections(d)
    ref = np.stack([rope.apply_mrope(x[:, h], co, theta(d), rope.axis_of_pair(sec)) for h in range(3)], 1)
    assert np.allclose(batch.norm_rope(x, None, 0, co, sec, theta(d)), ref, atol=1e-12)
    y = batch.norm_rope(x, np.full(d, 2.0), 0.0, co, sec, theta(d))
    assert np.allclose((y * y).mean(-1), 4.0)  # a rotation keeps the norm, the weight doubles it
    zero = batch.norm_rope(x, np.ones(d), 1e-6, co * 0, sec, theta(d))
    assert np.allclose(zero, x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6))


def test_attention_of_a_chain_is_the_selective_attention_of_the_last_rows():
    rng = np.random.default_rng(2)
    t, n, page, d = 37, 5, 8, 16
    k, v, q = (rng.standard_normal(s) for s in ((2, t, d), (2, t, d), (n, 4, d)))
    pool_k, pool_v = (np.zeros((5, 1, 2, page, d)) for _ in range(2))
    order = [3, 0, 4, 1, 2]
    for j in range(t):
        pool_k[order[j // page], 0, :, j % page], pool_v[order[j // page], 0, :, j % page] = k[:, j], v[:, j]
    out, lse = np.empty((n, 4, d)), np.empty((n, 4))
    batch.attend(q, pool_k, pool_v, 0, [t - n], [0, n], [order], None, out, lse)
    for r in range(n):
        for h in range(4):
            s = k[h // 2, :t - n + r + 1] @ q[r, h] / 4.0
            p = np.exp(s - s.max())
            assert np.allclose(out[r, h], p @ v[h // 2, :t - n + r + 1] / p.sum())
            assert np.isclose(lse[r, h], np.log(p.sum()) + s.max())
    # a row that sees nothing
    batch.attend(q, pool_k, pool_v, 0, [0], [0, 2], [order], [0, 2], out, lse)
    assert (out[0] == 0).all() and (lse[0] == -np.inf).all()
    assert np.allclose(out[1], v[:, 1][[0, 0, 1, 1]])


def test_commit_moves_rows_in_order():
    p = np.arange(6 * 1 * 1 * 4 * 1).reshape(6, 1, 1, 4, 1).copy()
    table = [[2, 5, 0]]
    flat = lambda: [int(p[table[0][j // 4], 0, 0, j % 4, 0]) for j in range(12)]
    before = flat()
    assert batch.commit([p], (0, 1), [3], [7], table, [[0, 2, 3, 6]], [4]) == [7]
    assert flat() == before[:3] + [before[3], before[5], before[6], before[9]] + before[7:]
    assert batch.commit([p], (0, 1), [3], [7], table, [[0, 2, 2, 6]], [4]) == [5]
    assert batch.commit([p], (0, 1), [3], [7], table, [[0, 7, 8, 9]], [4]) == [4]
