"""Verification with weights so small that the product of their sum and the random number is below fp32's normal numbers:
the border still falls where 64 bits put it.  Weights are whole numbers of 2^e, so that fp64 has sums and borders exactly."""
import numpy as np
import pytest

from oracle import chunk
from tests.gpu_helpers import torch_mod
from tests.test_gpu_tree import _expected, _same, _verify
from tests.test_gpu_verify import _check_verify

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _weights(rng, n, V, e, most):
    return (rng.integers(0, most, (n, V)) * 2.0 ** e).astype(np.float32)


@pytest.mark.parametrize("ns,V", [([40] * 60, 40), ([300], 517), ([3], 30001), ([300] * 12, 10007)])
@pytest.mark.parametrize("e", [-149, -140, -126, -100])
def test_tree(fp, ns, V, e):
    """A warp, a CTA and a cluster a row, and (the last) one row after the other: roots alone, each drawn from its own row."""
    rng = np.random.default_rng(V - e)
    N = sum(ns)
    p = _weights(rng, N, V, e, 4)
    p[:, V // 2] = 2.0 ** e
    u = rng.random(N).astype(np.float32)
    cu = np.concatenate([[0], np.cumsum(ns)])
    parent, tokens = np.full(N, -1, np.int32), np.full(N, -1, np.int32)
    for b in range(len(ns)):  # chains along what is drawn, so that every row's border counts
        for i in range(cu[b], cu[b + 1] - 1):
            parent[i + 1], tokens[i + 1] = i - cu[b], chunk.draw(p[i].astype(np.float64), float(u[i]))
    got = _verify(fp, p, cu, parent, tokens, u)
    _same(got, _expected(p, cu, parent, tokens, u))
    assert got[2].tolist() == ns


@pytest.mark.parametrize("e", [-149, -140, -126, -100])
@pytest.mark.parametrize("with_q", [False, True])
def test_draft(fp, e, with_q):
    """The draw behind a refused draft, and behind the last."""
    rng = np.random.default_rng(-e)
    B, V = 200, 501
    cu = np.arange(B + 1, dtype=np.int32) * 2
    p = _weights(rng, 2 * B, V, e, 4)
    p[:, 250] = 2.0 ** e
    q = _weights(rng, 2 * B, V, e, 3) if with_q else None
    tokens = rng.integers(0, V, 2 * B).astype(np.int32)
    u, r = np.full(2 * B, 0.9375, np.float32), rng.random(B).astype(np.float32)
    _check_verify(fp, p, q, tokens, u, r, cu)
