"""Beam selection with finite values that ban tokens, and rows whose largest logit is beyond 2^30 either way, against the
oracle.  Tolerances as in tests/test_gpu_beam_large.py up to 2^30; beyond it neighbours are 128 apart or more, so only the
logits equal to the largest count, which takes the place of the integer k: 2^-19 again.
"""
import numpy as np
import pytest

from tests.gpu_helpers import torch_mod
from tests.test_gpu_beam_large import _compare
from tests.test_gpu_beams import _select

pytestmark = pytest.mark.gpu

F32 = float(np.finfo(np.float32).max)
BF16 = 2.0 ** 127 * (2 - 2.0 ** -7)
MASKS = [-F32, -BF16, -1e38, -1e30, -1e15, -1e10, -1e9, -1e4]


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _banned(rng, how, V, W):
    t = np.arange(V)
    if how == "strips":  # whole shares of 128 tokens
        return (t // 128) % 16 % 5 == 3
    if how == "behind":
        return t >= min(V - W, V // 2 + 1)
    if how == "before":
        return t < V - W - 40
    keep = rng.choice(V, 2 * W, replace=False)  # "few" stay
    return ~np.isin(t, keep)


@pytest.mark.parametrize("how", ["strips", "behind", "before", "few"])
@pytest.mark.parametrize("B,W,V", [(2, 4, 32000), (1, 8, 128001), (3, 2, 5000), (1, 32, 70001), (2, 5, 16385), (1, 1, 300000)])
def test_select_beside_finite_bans(fp, how, B, W, V):
    rng = np.random.default_rng(V + len(how))
    for i, mask in enumerate(MASKS):
        x = (3 * rng.normal(size=(B * W, V))).astype(np.float32)
        x[:, _banned(rng, how, V, W)] = mask
        score = (-6 * rng.random(B * W)).astype(np.float32)
        _compare(_select(fp, x, B, W, score), x, B, W, score)
        if i % 3 == 0:
            done = np.arange(B * W) % 3 == 1
            _compare(_select(fp, x, B, W, score, done, 2, offset=1), x, B, W, score, done, 2)


def test_select_beside_bans_of_every_kind(fp):
    """Bans that differ from place to place, -inf among them, and beams with and without them."""
    rng = np.random.default_rng(5)
    B, W, V = 2, 6, 40000
    x = (3 * rng.normal(size=(B * W, V))).astype(np.float32)
    kinds = np.array(MASKS + [-np.inf], np.float32)
    ban = rng.integers(0, 2, (B * W, (V + 127) // 128)).repeat(128, 1)[:, :V].astype(bool)
    ban[::3] = False
    x = np.where(ban, kinds[rng.integers(0, len(kinds), x.shape)], x)
    score = (-4 * rng.random(B * W)).astype(np.float32)
    _compare(_select(fp, x, B, W, score), x, B, W, score)


@pytest.mark.parametrize("mask", MASKS + [-(2.0 ** 30), -(2.0 ** 30 - 64), -(2.0 ** 30 + 128)])
@pytest.mark.parametrize("W,V", [(4, 32000), (32, 700), (3, 50), (2, 70001)])
def test_select_of_banned_rows_only(fp, mask, W, V):
    """Every token banned alike: as probable as any other, and taken in the tokens' order."""
    rng = np.random.default_rng(W)
    x = np.full((2 * W, V), mask, np.float32)
    x[W, 0] = -np.inf
    score = (-5 * rng.random(2 * W)).astype(np.float32)
    score[1:W] = -np.inf
    got = _select(fp, x, 2, W, score)
    _compare(got, x, 2, W, score)
    assert got[0][:W].tolist() == [0] * W and got[1][:W].tolist() == list(range(W))


@pytest.mark.parametrize("mask", MASKS)
def test_select_falls_back_on_banned_tokens(fp, mask):
    """Fewer tokens than places: the lowest banned ones follow, with the ban as their score."""
    W, V = 8, 20000
    x = np.full((W, V), mask, np.float32)
    x[:, [17, 4000, 19999]] = [1.0, 3.0, 2.0]
    score = np.where(np.arange(W) == 2, -1.5, -np.inf).astype(np.float32)
    got = _select(fp, x, 1, W, score)
    _compare(got, x, 1, W, score)
    assert got[1].tolist() == [4000, 19999, 17, 0, 1, 2, 3, 4]


def test_select_leaves_out_what_fp32_does_not_hold(fp):
    """A candidate whose score would be below the least fp32 is none; one that rounds to the least is one."""
    W, V = 4, 9000
    for top, places in ((1e33, 1), (5e30, 4)):
        x = np.full((W, V), -F32, np.float32)
        x[:, 77] = top
        score = np.array([0.0, -np.inf, -np.inf, -np.inf], np.float32)
        got = _select(fp, x, 1, W, score)
        _compare(got, x, 1, W, score)
        assert got[1].tolist() == [77, 0, 1, 2][:places] + [-1] * (W - places)


@pytest.mark.parametrize("top", [2.0 ** 30, 2.0 ** 30 + 128, 1e10, 1e15, 1e30, 1e38, BF16, F32])
@pytest.mark.parametrize("sign", [1, -1])
def test_select_of_rows_far_from_zero(fp, top, sign):
    """Rows whose largest is beyond 2^30 either way: it counts as often as it is there, whatever stands beside it."""
    rng = np.random.default_rng(7)
    W, V = 5, 50001
    m = np.float32(sign * top)
    x = np.empty((W, V), np.float32)
    low = m if m == -np.float32(F32) else np.nextafter(m, np.float32(-np.inf))
    x[0] = -np.inf
    x[0, 4:300:3] = m
    x[1] = low
    x[1, [9, 49999]] = m
    x[2] = m
    x[3] = np.where(rng.random(V) < 0.5, m, -np.float32(F32))
    x[4] = (np.float32(min(m, 0)) + 3 * rng.normal(size=V)).astype(np.float32)
    x[4, 11] = m
    for live in ([0], [1], [2], [3], [4], [0, 1, 2, 3, 4]):
        score = np.full(W, -np.inf, np.float32)
        score[live] = (-9 * rng.random(len(live))).astype(np.float32)
        _compare(_select(fp, x, 1, W, score), x, 1, W, score)


@pytest.mark.parametrize("at", [2.0 ** 30, -(2.0 ** 30)])
def test_select_across_the_border(fp, at):
    """Largest values just above, on and just below 2^30 in different shares of a row."""
    W, V = 3, 40000
    base = np.float32(at)
    x = np.full((W, V), base - np.float32(64 if at > 0 else 128), np.float32)
    x[0, 20000] = base
    x[1, 100:140] = base + np.float32(128 if at > 0 else 64)
    x[1, 30000:31000] = base
    x[2, ::2] = base + np.float32(256 if at > 0 else 128)
    score = np.array([-1.0, -3.0, -8.0], np.float32)
    _compare(_select(fp, x, 1, W, score), x, 1, W, score)


def test_select_reports_infinities_beside_bans(fp):
    """+inf and NaN beside low finite values are reported as ever."""
    rng = np.random.default_rng(1)
    W, V = 2, 40000
    for what in (np.nan, np.inf):
        for mask in MASKS:
            x = (3 * rng.normal(size=(W, V))).astype(np.float32)
            x[:, 256:] = mask
            x[0, 39999] = what
            got = _select(fp, x, 1, W, np.array([-1.0, -2.0], np.float32))
            assert got[4] == 1 and got[0].tolist() == [1, 1]
