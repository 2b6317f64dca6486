"""Sizes of the attention of a chunk that its 32-bit places within a unit's output do not hold: refused on the host,
before any CUDA call, so this runs without a GPU."""
import pytest

from tests.test_chunk_abi import A, UNSUPPORTED, code, fp, view  # noqa: F401


@pytest.mark.parametrize("hd,Hkv,G", [(128, 65536, 1),
                                       (64, 131072, 1), (128, 65536, 2), (128, 65536, 128), (128, 83887, 100)])
def test_output_rows_beyond_32_bits_are_refused(fp, hd, Hkv, G):  # noqa: F811
    """A unit of T tokens (twice the largest power of two up to 128 / G) writes elements 0 .. T H hd - 1 from its first
    row on."""
    H = Hkv * G

    def call(H, Hkv):
        kv = view(fp, hd=hd, Hkv=Hkv, pages=4)
        return code(lambda: fp.fp_op_attention_chunk(A, H * hd, 1, 1, H, kv, A, A, 1, 16, A, None, 0))

    T = 2 << ((128 // G).bit_length() - 1)
    assert T * H * hd >= 2 ** 31 > T * (H - G) * hd
    assert call(H, Hkv) == UNSUPPORTED
    assert call(H - G, Hkv - 1) == -1  # fits: the next check, a workspace of NULL
