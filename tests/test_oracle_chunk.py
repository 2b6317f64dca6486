"""The oracle of probabilities and draft verification, pinned by closed forms and by the distribution it has to give."""
import numpy as np

from oracle import chunk


def test_probabilities_closed_forms():
    x = np.log(np.array([[1.0, 2.0, 5.0]]))
    assert np.allclose(chunk.probabilities(x), [[0.125, 0.25, 0.625]])
    assert np.allclose(chunk.probabilities(x, [0.5]), np.array([[1, 4, 25]]) / 30)
    assert chunk.probabilities(np.array([[3.0, 7, 7, 1]]), [0.0]).tolist() == [[0, 1, 0, 0]]
    assert chunk.probabilities(np.full((1, 4), -np.inf)).tolist() == [[0, 0, 0, 0]]
    assert chunk.probabilities(x, [-1.0]).tolist() == [[0, 0, 0]]


def test_draw_borders():
    w = np.array([0.0, 0.25, 0.25, 0.0, 0.5])
    assert [chunk.draw(w, r) for r in (0.0, 0.2499, 0.25, 0.4999, 0.5, 0.9999, 1.0)] == [1, 1, 2, 2, 4, 4, 4]


def test_verify_hand_worked():
    p = np.array([[0.5, 0.5, 0.0], [0.2, 0.2, 0.6], [0.1, 0.2, 0.7]])
    q = np.array([[0.25, 0.75, 0.0], [0.8, 0.1, 0.1], [0.0, 0.0, 0.0]])
    # draft 1: 0.6 * 0.75 < 0.5; draft 0: 0.5 * 0.8 >= 0.2 refused; then max(0, p - q) = (0, .1, .5)
    assert chunk.verify(p, q, [9, 1, 0], [0.6, 0.5, 0.0], 0.1) == ([1, 1], True)
    assert chunk.verify(p, q, [9, 1, 0], [0.6, 0.5, 0.0], 0.2) == ([1, 2], True)
    # all accepted: one more from the last row
    assert chunk.verify(p, q, [9, 1, 0], [0.6, 0.2, 0.0], 0.05) == ([1, 0, 0], True)
    # certain drafts: accepted with probability p, refused ones never drawn
    assert chunk.verify(p, None, [9, 1, 2], [0.4, 0.7, 0.0], 0.999) == ([1, 1], True)
    assert chunk.verify(p, None, [9, 7, 2], [0.4, 0.7, 0.0], 0.0) == ([0], False)


def test_verify_gives_the_target_distribution():
    """One draft from q, verified: what is emitted first is distributed as p (the method's theorem)."""
    rng = np.random.default_rng(3)
    p = np.array([[0.1, 0.2, 0.3, 0.4]] * 2)
    q = np.array([[0.4, 0.3, 0.2, 0.1]] * 2)
    n = 20000
    seen = np.zeros(4)
    for d, u, r in zip(rng.choice(4, n, p=q[0]), rng.random(n), rng.random(n)):
        seen[chunk.verify(p, q, [0, d], [u, 0.0], r)[0][0]] += 1
    assert np.all(np.abs(seen / n - p[0]) < 5 * np.sqrt(p[0] * (1 - p[0]) / n))
