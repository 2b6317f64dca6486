"""Tree attention of sequences with more rows than max_new: what the first max_new rows are."""
import numpy as np
import pytest

from oracle import several
from tests.gpu_helpers import torch_mod
from tests.test_gpu_tree import Trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _check_cut(c, q, got, seen, most):
    """The first `most` rows of each sequence see the prefix and, of one another, what their masks say; the rest is left."""
    cut = Trees.__new__(Trees)
    cut.__dict__.update(c.__dict__)
    untouched = np.ones(c.N, bool)
    for b, (n, p) in enumerate(c.seqs):
        n1, r = min(n, most), slice(int(c.cu[b]), int(c.cu[b]) + min(n, most))
        untouched[r] = False
        one = Trees.__new__(Trees)
        one.__dict__.update(c.__dict__)
        one.seqs, one.cu, one.N = [(n1, p)], np.array([0, n1]), n1
        one.table = c.table[b : b + 1]
        one.check(q[r], got[r], seen=[[{j for j in s if j < n1} for s in seen[b][:n1]]])
    assert np.all(got[untouched] == 0x4321)


@pytest.mark.parametrize("kvq", [0, 1])
@pytest.mark.parametrize("most", [1, 4, 33, 39])
def test_rows_within_max_new(fp, kvq, most):
    seqs = [(6, 0), (9, 60), (40, 30), (150, 700), (1, 5)]
    c = Trees(fp, kvq, 128, 8, 2, seqs, 29, words=5)
    q = c.queries(9)
    got, err = c.attend(q, max_new=most)
    assert err == 1
    _check_cut(c, q, got, c.seen, most)


@pytest.mark.parametrize("kvq", [0, 1])
def test_rows_within_max_new_of_any_mask(fp, kvq):
    """Masks that name rows behind the bound: those are not seen."""
    rng = np.random.default_rng(3)
    c = Trees(fp, kvq, 64, 4, 4, [(20, 0), (70, 100), (3, 9)], 31, words=3)
    seen = [[set(np.nonzero(rng.random(n) < 0.5)[0].tolist()) | {i % 4} for i in range(n)] for n, _ in c.seqs]
    m = np.zeros((c.N, 3), np.uint32)
    for b, s in enumerate(seen):
        m[c.cu[b] : c.cu[b + 1]] = several.words(s, 3)
    q = c.queries(9)
    got, err = c.attend(q, mask=m, max_new=17)
    assert err == 1
    _check_cut(c, q, got, seen, 17)
