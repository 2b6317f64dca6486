"""NaN and infinite scores in the attention of a chunk: the rows that see one are NaN, wherever the batch's lengths cut
their unit, and every other row keeps its bits."""
import numpy as np
import pytest

from oracle import quant
from tests.gpu_helpers import dev, torch_mod
from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu

NAN, INF = 0x7FC0, 0x7F80  # bf16


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


# hd, H, Hkv, (rows, position): a unit of one CTA, of two query tiles; one tile cut over 10 CTAs, and over 59 (its parts
# are added in two turns); two tiles cut; many sequences, of which some are cut
SHAPES = [
    (128, 8, 1, [(3, 20)]),
    (64, 4, 4, [(200, 7)]),
    (128, 8, 1, [(4, 5000)]),
    (128, 8, 1, [(4, 30000)]),
    (64, 8, 1, [(32, 3000)]),
    (128, 10, 2, [(5, 700), (40, 900), (1, 2000)] * 3),
]


def _expect(c, clean, got, bad):
    """bad [N, H]: those heads of those rows are NaN throughout, all others as they were."""
    g = quant.bf16_to_f32(got).reshape(c.N, c.H, c.hd)
    assert np.all(np.isnan(g[bad])), np.argwhere(bad & ~np.isnan(g).all(-1))[:5]
    same = (got == clean).reshape(c.N, c.H, c.hd).all(-1)
    assert np.all(same | bad), np.argwhere(~same & ~bad)[:5]


@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("kvq", [0, 1])
def test_a_query_that_is_not_finite(fp, kvq, shape, value):
    """One element of a query head: its scores are NaN, or infinities of both signs, and so is its softmax."""
    hd, H, Hkv, seqs = SHAPES[shape]
    c = Batch(fp, kvq, hd, H, Hkv, seqs, 71 + shape)
    q = c.queries(3)
    clean, err = c.attend(q)
    assert err == 0
    c.check(q, clean)
    bad = np.zeros((c.N, H), bool)
    for b, (n, p) in enumerate(seqs):
        r, h, x = int(c.cu[b]) + n // 2, (3 * b + 1) % H, (5 * b) % hd
        k = c.cached("k", b, p + n // 2 + 1)[:, h // (H // Hkv), x]
        assert np.any(k > 0)  # a score of +inf, whose softmax is NaN
        q[r, h * hd + x] = value
        bad[r, h] = True
    got, err = c.attend(q)
    assert err == 0
    _expect(c, clean, got, bad)


@pytest.mark.parametrize("back", [0, 1, 300])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("kvq", [0, 1])
def test_a_key_that_is_nan(fp, kvq, shape, back):
    """The key `back` positions before each sequence's last one (an int8 cache: its scale), of one KV head: NaN in the
    rows that see it, nothing in the rows before it."""
    hd, H, Hkv, seqs = SHAPES[shape]
    c = Batch(fp, kvq, hd, H, Hkv, seqs, 81 + shape)
    q = c.queries(4)
    clean, err = c.attend(q)
    assert err == 0
    bad = np.zeros((c.N, H), bool)
    for b, (n, p) in enumerate(seqs):
        t, kh = max(0, p + n - 1 - back), b % Hkv
        page, slot = c.table[b, t // 16], t % 16
        if kvq:
            c.data["ks"][page, kh, slot] = np.nan
        else:
            c.data["k"][page, kh, slot] = NAN
        G = H // Hkv
        bad[int(c.cu[b]) + max(0, t - p):int(c.cu[b]) + n, kh * G:(kh + 1) * G] = True
    for w in c.data:
        c.dev[w] = dev(c.data[w])
    c.view = c.make_view(c.table)
    got, err = c.attend(q)
    assert err == 0
    _expect(c, clean, got, bad)


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("kvq", [0, 1])
def test_a_row_whose_scores_are_all_minus_infinity(fp, kvq, shape):
    """No key has weight: zeros, as for a row without keys, cut or not."""
    hd, H, Hkv, seqs = SHAPES[shape]
    c = Batch(fp, kvq, hd, H, Hkv, seqs, 91 + shape)
    c.data["k"][..., 9] = -5 if kvq else 0xC000  # (bf16: -2)
    c.dev["k"] = dev(c.data["k"])
    c.view = c.make_view(c.table)
    q = c.queries(5)
    clean, err = c.attend(q)
    assert err == 0
    rows = c.cu[:-1]
    q[rows, 2 * hd + 9] = INF
    got, err = c.attend(q)
    assert err == 0
    assert np.all(got.reshape(c.N, H, hd)[rows, 2] & 0x7FFF == 0)
    rest = np.ones((c.N, H), bool)
    rest[rows, 2] = False
    assert np.array_equal(got.reshape(c.N, H, hd)[rest], clean.reshape(c.N, H, hd)[rest])
