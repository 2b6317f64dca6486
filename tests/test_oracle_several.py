"""Pins of the oracle's trees and beams: closed forms, brute force, worked examples."""
import itertools

import numpy as np
import pytest

from oracle import chunk, several
from oracle import model as M


def test_plan_of_a_worked_tree():
    #        0 - 1 - 3
    #         \- 2 - 4 - 5
    depth, seen, good = several.plan([-1, 0, 0, 1, 2, 4])
    assert good and depth == [0, 1, 1, 2, 2, 3]
    assert seen == [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {0, 2, 4}, {0, 2, 4, 5}]
    assert several.words(seen, 1)[:, 0].tolist() == [1, 3, 5, 11, 21, 53]
    assert several.plan([0, 5, -2])[::2] == ([0, 0, 0], False)


def test_words_of_rows_beyond_32():
    depth, seen, _ = several.plan([-1] + list(range(69)))
    w = several.words(seen, 3)
    assert depth[-1] == 69 and w[69].tolist() == [0xFFFFFFFF, 0xFFFFFFFF, 0x3F] and w[31].tolist() == [0xFFFFFFFF, 0, 0]


def test_attention_of_a_chain_is_the_chunk_s():
    rng = np.random.default_rng(0)
    n, p, H, Hkv, hd = 5, 7, 4, 2, 8
    q, k, v = rng.normal(size=(n, H, hd)), rng.normal(size=(p + n, Hkv, hd)), rng.normal(size=(p + n, Hkv, hd))
    visible = np.arange(p + n)[None] <= p + np.arange(n)[:, None]
    assert np.allclose(several.attention(q, visible, k, v), M.attention(q, p + np.arange(n), k, v), atol=1e-12)
    assert np.all(several.attention(q, np.zeros_like(visible), k, v) == 0)


def test_a_verified_tree_is_distributed_as_the_target():
    """Over a grid of u the first two tokens have the target's probabilities, on whatever branch they lie."""
    p = np.array([[0.5, 0.25, 0.25], [0.25, 0.25, 0.5], [0.0, 0.75, 0.25]])
    parent, tokens = [-1, 0, 0], [9, 0, 2]
    count = {}
    grid = (np.arange(8) + 0.5) / 8
    for u0, u1, u2 in itertools.product(grid, grid, grid):
        path, out, good = several.verify(p, parent, tokens, [u0, u1, u2])
        assert good and len(path) == len(out)
        count[tuple(out)] = count.get(tuple(out), 0) + 1 / 512
    assert count == {(0, 0): 0.125, (0, 1): 0.125, (0, 2): 0.25, (1,): 0.25, (2, 1): 0.1875, (2, 2): 0.0625}


def test_a_verified_chain_is_the_draft_verification_of_certain_drafts():
    """Accepting t with probability p(t), then drawing without t, is drawing: the accepted lengths agree in distribution
    (a chain of two, counted over a grid)."""
    p = np.array([[0.5, 0.5], [0.25, 0.75], [1.0, 0.0]])
    tokens = [0, 1, 0]
    grid = (np.arange(16) + 0.5) / 16
    a, b = np.zeros(4), np.zeros(4)
    for u0, u1 in itertools.product(grid, grid):
        a[len(several.verify(p, [-1, 0, 1], tokens, [u0, u1, 0.5])[1])] += 1
        b[len(chunk.verify(p, None, tokens, [u0, u1, 0.5], 0.5)[0])] += 1
    assert np.array_equal(a, b)


@pytest.mark.parametrize("W,V", [(1, 3), (2, 4), (3, 5), (4, 2)])
def test_selection_by_brute_force(W, V):
    rng = np.random.default_rng(W * 10 + V)
    x, score = rng.integers(-3, 3, (W, V)).astype(float), -rng.random(W)
    done = np.arange(W) % 3 == 2
    got, good = several.select(x, score, done, 1)
    assert good
    every = []
    for w in range(W):
        if done[w]:
            every.append((-score[w], w, 1))
            continue
        z = np.exp(x[w]) / np.exp(x[w]).sum()
        every += [(-(score[w] + np.log(z[t])), w, t) for t in range(V)]
    every = sorted((round(v, 12), w, t) for v, w, t in every)[:W]
    assert [(w, t) for w, t, _, _ in got] == [(w, t) for _, w, t in every]
    assert np.allclose([s for _, _, s, _ in got], [-v for v, _, _ in every])
    assert [d for _, _, _, d in got] == [int(done[w] or t == 1) for _, w, t in every]


def test_selection_without_enough_candidates():
    x = np.array([[0.0, -np.inf], [np.nan, 0.0], [5.0, 5.0]])
    got, good = several.select(x, [-1.0, -1.0, -np.inf], [0, 0, 0], -1)
    assert not good and got == [(0, 0, -1.0, 0), (-1, -1, -np.inf, 0), (-1, -1, -np.inf, 0)]


def test_reordering_of_a_worked_group():
    table = [[10, 11, 12], [20, 21, 22], [30, 31, 32], [40, 41, 42]]
    new, copies, good = several.reorder(table, 21, [2, 2, 0, 2])
    assert good
    # 2's first child keeps page 31, the others take those of 1 and 3, which have no children
    assert new.tolist() == [[30, 31, 12], [30, 21, 22], [10, 11, 32], [30, 41, 42]]
    assert copies == [(-1, -1, 0), (31, 21, 5), (-1, -1, 0), (31, 41, 5)]
    new, copies, _ = several.reorder(table, 32, [3, 3, 3, 3])
    assert new.tolist() == [[40, 41, 12], [40, 41, 22], [40, 41, 32], [40, 41, 42]] and copies == [(-1, -1, 0)] * 4
    new, copies, good = several.reorder(table, 5, [1, -1, 9, 1])
    assert not good and new.tolist() == [[20, 11, 12], [10, 21, 22], [30, 31, 32], [40, 41, 42]]
    assert copies == [(-1, -1, 0)] * 3 + [(20, 40, 5)]


@pytest.mark.parametrize("seed", range(20))
def test_reordering_keeps_every_beam_s_history(seed):
    """Steps of reordering, copying and appending: each beam's table leads to its own tokens, as plain lists have them."""
    rng = np.random.default_rng(seed)
    W, page, pps = 4, 4, 5
    table = rng.permutation(W * pps).reshape(W, pps)
    cells = {}
    texts = [[] for _ in range(W)]
    for step in range(pps * page):
        parent = rng.integers(0, W, W)
        table, copies, good = several.reorder(table, step, parent, page)
        assert good
        reads, writes = {c[0] for c in copies if c[2]}, [c[1] for c in copies if c[2]]
        assert len(set(writes)) == len(writes) and not reads & set(writes)
        for a, b, n in copies:
            for i in range(n):
                cells[b, i] = cells[a, i]
        texts = [list(texts[p]) for p in parent]
        for w in range(W):
            texts[w].append((step, w))
            cells[table[w, step // page], step % page] = (step, w)
        for w in range(W):
            assert [cells[table[w, i // page], i % page] for i in range(step + 1)] == texts[w]
