"""Chunked serving for batches of many sequences, most of them without rows."""
import numpy as np
import pytest

import synth
from oracle import model as M
from oracle import quant
from tests.gpu_helpers import torch_mod
from tests.test_gpu_chunk import BASE, Batch, _append

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _seqs(B, seed):
    rng = np.random.default_rng(seed)
    n = rng.integers(0, 4, B) * (rng.random(B) < 0.4)
    n[[0, B - 1]] = 0  # none at the ends
    return [(int(a), int(p)) for a, p in zip(n, rng.integers(0, 120, B))]


@pytest.mark.parametrize("B", [33, 1024, 1025, 1500])
@pytest.mark.parametrize("kvq", [0, 1])
def test_many_sequences(fp, kvq, B):
    """The sequence of a row is found among thousands: values read back are those of its own row, rotations those of its
    position; and its attention is over its own keys."""
    hd, H, Hkv = 64, 4, 2
    c = Batch(fp, kvq, hd, H, Hkv, _seqs(B, B), 141, lead=2, tail=3)
    qkv = synth.uniform_bf16(142, B, (c.N, (H + 2 * Hkv) * hd), -3, 3)
    q, k, v, err = _append(c, qkv)
    assert err == 0
    own = np.zeros(c.N, bool)
    x = qkv.reshape(c.N, H + 2 * Hkv, hd)
    f = quant.bf16_to_f32(x).astype(np.float64)
    for b, (n, p) in enumerate(c.seqs):
        r = slice(int(c.cu[b]), int(c.cu[b]) + n)
        own[r] = True
        if n == 0:
            continue
        ref = M.rope(f[r, :H], p + np.arange(n), BASE)
        got = quant.bf16_to_f32(q[r, : H * hd]).reshape(n, H, hd)
        # one bf16 rounding, three of fp32 and the table's on the pair (components up to 3)
        assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -22 * 3 * np.sqrt(2))
        want = x[r, H + Hkv:]
        if kvq:
            codes, s = quant.quantize_kv_int8(want)
            want = synth.f32_to_bf16_bits(codes.astype(np.float32) * s[..., None])
        assert np.array_equal(v[r, : Hkv * hd].reshape(n, Hkv, hd), want)
    assert np.all(q[~own] == 0x4321) and np.all(k[~own] == 0x4321) and np.all(v[~own] == 0x4321)
    c = Batch(fp, kvq, hd, H, Hkv, c.seqs, 143, lead=2, tail=3)
    q = c.queries(9)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)
