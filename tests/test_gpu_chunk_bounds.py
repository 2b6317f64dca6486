"""Lengths beyond the bounds of the attention of a chunk: what the rows that are still computed come to."""
import numpy as np
import pytest

from oracle import model as M
from oracle import quant
from tests.gpu_helpers import torch_mod
from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _close(c, q, got, rows, b, upto):
    """Rows `rows` of sequence b, row i over keys 0 .. upto[i]-1 (none: zeros); the tolerance of Batch.check."""
    H, hd = c.H, c.hd
    upto = np.asarray(upto)
    n = max(int(upto.max()), 1)
    k, v = c.cached("k", b, n), c.cached("v", b, n)
    x = quant.bf16_to_f32(q[rows, : H * hd]).astype(np.float64).reshape(-1, H, hd)
    o = quant.bf16_to_f32(got[rows]).astype(np.float64).reshape(-1, H, hd)
    some = upto > 0
    ref, mass = (M.attention(x[some], upto[some] - 1, k, y) for y in (v, np.abs(v)))
    assert np.all(np.abs(o[some] - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * mass + 1e-30)
    assert np.all(o[~some] == 0)


@pytest.mark.parametrize("hd,H,Hkv", [(128, 8, 2), (64, 4, 4), (128, 16, 1)])
@pytest.mark.parametrize("kvq", [0, 1])
def test_rows_before_max_new_are_computed(fp, kvq, hd, H, Hkv):
    """Sequences with more rows than max_new: the first max_new as ever, the others as they were."""
    seqs = [(6, 40), (9, 64), (2, 30), (70, 400)]
    c = Batch(fp, kvq, hd, H, Hkv, seqs, 111)
    q = c.queries(7)
    for most in (1, 4, 33):
        got, err = c.attend(q, max_new=most)
        assert err == 1
        for b, (n, p) in enumerate(seqs):
            m, r = min(n, most), int(c.cu[b])
            _close(c, q, got, slice(r, r + m), b, p + 1 + np.arange(m))
            assert np.all(got[r + m:r + n] == 0x4321)


@pytest.mark.parametrize("pos", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30, 1000, -1, -30, -2 ** 31])
@pytest.mark.parametrize("kvq", [0, 1])
def test_positions_far_outside(fp, kvq, pos):
    """A position behind max_len: the rows see the max_len keys that there are; a negative one: none."""
    c = Batch(fp, kvq, 128, 8, 2, [(5, 40), (50, 300), (3, 20)], 113)
    q = c.queries(8)
    at = c.pos.copy()
    at[1] = pos
    got, err = c.attend(q, pos=at)
    assert err == 1
    upto = np.clip(pos + 1 + np.arange(50, dtype=np.int64), 0, c.max_len)
    _close(c, q, got, slice(5, 55), 1, upto)
    c.check(q, got, only={0, 2})
