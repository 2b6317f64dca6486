"""Beam selection of rows whose largest logit is between 2^23 and 2^30 either way, against the oracle.

Tolerances as in tests/test_gpu_beams.py: a score is off by 2^-24 of it and the normaliser's 2^-19.  The normaliser is
(k + log2 s) ln 2 with an integer k, and what it holds in pairs of fp32 is about as large as the row's largest logit m:
each of its products and sums keeps 2^-47 |m| or better, ln 2 in two parts 2^-53 |m|, and the exponents, of up to
2^-23 |m|, are rounded twice, 2^-46 |m|: together less than 2^-44 |m|.
"""
import numpy as np
import pytest

from oracle import several
from tests.gpu_helpers import torch_mod
from tests.test_gpu_beams import LSE, _select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _compare(got, x, B, W, score, done=None, end=-1, err=0):
    """All places: the oracle's candidate (another of a value that is not told apart, where beams differ) and its score."""
    par, tok, new, nd, e = got
    done = np.zeros(B * W, int) if done is None else np.array(done)
    for b in range(B):
        r = slice(b * W, b * W + W)
        want, good = several.select(x[r], score[r], done[r], end)
        assert good
        top = np.abs(np.max(np.where(np.isnan(x[r]), -np.inf, x[r]), -1).astype(np.float64))
        most = max([m for m in top if m <= 2.0 ** 30], default=0.0)
        tol = max(LSE, 2.0 ** -44 * most)
        for c, (pw, pt, ps, pd) in enumerate(want):
            o = b * W + c
            if pw < 0:
                assert (par[o], tok[o], new[o], nd[o]) == (-1, -1, -np.inf, 0), (b, c, par[o], tok[o], new[o])
                continue
            assert abs(float(new[o]) - ps) <= 2.0 ** -24 * abs(ps) + tol, (b, c, new[o], want[c])
            near = any(q[0] != pw and abs(ps - q[2]) <= 2.0 ** -23 * abs(ps) + 2 * tol for q in want)
            if not near and c < W - 1 or W == 1:
                assert (par[o], tok[o]) == (pw, pt), (b, c, par[o], tok[o], want[c])
            assert nd[o] == int(bool(done[b * W + par[o]]) or tok[o] == end)
    assert e == err


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("top", [2.0 ** 23, 3e7, 1e8, 123456789.0, 5e8, 1.07e9])
def test_select_of_large_rows(fp, top, sign):
    """One row alone, several of them, and beside ordinary ones."""
    rng = np.random.default_rng(int(top) % 1000)
    W, V = 4, 30001
    x = (sign * top + 40 * rng.normal(size=(W, V))).astype(np.float32)
    x[1] = (sign * top + 400 * rng.normal(size=V)).astype(np.float32)
    x[3] = (3 * rng.normal(size=V)).astype(np.float32)
    for live in ([0], [1], [0, 2], [0, 1, 2, 3]):
        score = np.full(W, -np.inf, np.float32)
        score[live] = (-9 * rng.random(len(live))).astype(np.float32)
        _compare(_select(fp, x, 1, W, score), x, 1, W, score)
