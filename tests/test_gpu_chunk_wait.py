"""The failure path of the attention of a chunk, without a fault: a wait that runs out ends in status 2, with every copy
and product in flight drained, and the next call is right again."""
import numpy as np
import pytest

from tests.gpu_helpers import empty, host, ptr, torch_mod
from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


@pytest.mark.parametrize("kvq", [0, 1])
def test_an_expired_wait_is_reported(fp, kvq):
    """The issuing warps give up at their first tile of values.  Units of one and of two tiles, several a CTA, whole and
    cut; after the tickets are zeroed again, as the interface asks, the same workspace serves the same batch."""
    c = Batch(fp, kvq, 128, 64, 8, [(5, 700), (40, 900), (1, 2000), (3, 20)] * 3, 101)
    q = c.queries(6)
    need = fp.fp_op_attention_chunk_workspace_bytes(c.B, c.H, c.Hkv, c.hd, c.max_new)
    ws = empty(need + 256)
    fp.fp_debug_set_wait_limit(0)
    try:
        _, err = c.attend(q, ws=ws)
    finally:
        fp.fp_debug_set_wait_limit(-1)
    assert err == 2
    at = -ptr(ws) % 256
    ws[at:at + 65536] = 0
    for _ in range(2):
        got, err = c.attend(q, ws=ws)
        assert err == 0
        c.check(q, got)
    assert not host(ws, np.uint8)[at:at + 65536].any()
