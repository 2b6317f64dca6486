"""Verification of drafted tokens: what lies behind the first refusal, and products that underflow."""
import numpy as np
import pytest

from oracle import chunk
from tests.gpu_helpers import torch_mod
from tests.test_gpu_verify import _check_verify

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


@pytest.mark.parametrize("onehot", [False, True])
@pytest.mark.parametrize("k,refused", [(3, 0), (5, 2), (31, 30), (40, 3), (40, 33), (70, 31), (70, 32)])
def test_padding_behind_the_first_refusal_is_not_looked_at(fp, k, refused, onehot):
    """Drafts of -1 behind the refused one are no error, however many; the first of them in the refused one's place is."""
    V = 64
    rng = np.random.default_rng(k + refused)
    p = chunk.probabilities(rng.standard_normal((2 * (k + 1), V))).astype(np.float32)
    q = None if onehot else p.copy()
    u = np.zeros(len(p), np.float32)  # u q < p: accepted
    u[refused] = 1.0                  # u q < p does not hold where q = p or 1: refused
    tokens = rng.integers(0, V, len(p)).astype(np.int32)
    tokens[refused + 2:k + 1] = -1
    r, cu = np.array([0.3, 0.6], np.float32), np.array([0, k + 1, 2 * (k + 1)])
    out, cnt = _check_verify(fp, p, q, tokens, u, r, cu)
    assert cnt.tolist() == [refused + 1, k + 1]
    tokens[refused + 1] = V
    _check_verify(fp, p, q, tokens, u, r, cu)  # (the oracle says: reported)


def test_products_that_underflow(fp):
    """u q < p where p is the fp32 next to u q, and what tells them apart is below the least fp32: accepted
    where the exact product is the smaller, refused where it is not."""
    rng = np.random.default_rng(6)
    V, want, parts = 8, [], []
    while len(want) < 64:
        u, qt = np.float32((1 + rng.random()) * 2.0 ** -126), np.float32(0.5 + rng.random() / 2)
        exact, pt = float(u) * float(qt), np.float32(float(u) * float(qt))
        if exact == float(pt) or (exact < float(pt)) != (len(want) % 2 == 0):
            continue
        want.append(exact < float(pt))
        p, q = np.full((2, V), 0.125, np.float32), np.full((2, V), 0.125, np.float32)
        p[0, 5], q[0, 5] = pt, qt
        parts.append((p, q, u))
    B = len(want)
    p, q = np.concatenate([x[0] for x in parts]), np.concatenate([x[1] for x in parts])
    u = np.zeros(2 * B, np.float32)
    u[::2] = [x[2] for x in parts]
    tokens = np.tile(np.array([0, 5], np.int32), B)
    out, cnt = _check_verify(fp, p, q, tokens, u, rng.random(B, dtype=np.float32), 2 * np.arange(B + 1))
    assert (cnt == 2).tolist() == want
