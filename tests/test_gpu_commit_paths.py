"""Commit of paths that hold entries below -1: no rows of their sequence, so the path ends there and is reported."""
import numpy as np
import pytest

from tests.gpu_helpers import torch_mod
from tests.test_gpu_tree import Trees, _commit, _committed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


@pytest.mark.parametrize("kvq", [0, 1])
@pytest.mark.parametrize("at", [0, 1, 33])
def test_commit_reports_entries_below_minus_one(fp, kvq, at):
    seqs = [(40, 10), (40, 3), (6, 20)]
    for entry in (-2, -5, -2 ** 31):
        c = Trees(fp, kvq, 128, 4, 2, seqs, 25)
        path = list(range(1, 36))
        got, err = _commit(c, c.flat([path[:at] + [entry] + path[at + 1 :], path[:at], [1, 4]]))
        assert err == 1, entry
        want = _committed(c, [path[:at], path[:at], [1, 4]])
        for w in want:
            assert np.array_equal(got[w].reshape(want[w].shape).view(np.uint8), want[w].view(np.uint8)), w


def test_commit_does_not_look_behind_an_end(fp):
    c = Trees(fp, 0, 128, 4, 2, [(40, 10)], 25)
    got, err = _commit(c, c.flat([[1, 3, -1, -7, 2] + [-9] * 35]))
    assert err == 0
    want = _committed(c, [[1, 3]])
    for w in want:
        assert np.array_equal(got[w].reshape(want[w].shape).view(np.uint8), want[w].view(np.uint8)), w
