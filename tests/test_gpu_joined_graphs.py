"""Calls that start early, captured where two streams join: they wait for both."""
import numpy as np
import pytest

import synth
from tests.gpu_helpers import dev, empty, host, ptr, torch_mod
from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("kvq", [0, 1])
def test_append_behind_two_streams(fp, graph, kvq):
    """A long product on one stream and one on another, then append, read back and attention: what the products wrote is
    what is appended, first and later times."""
    torch = torch_mod()
    c = Batch(fp, kvq, 128, 8, 2, [(60, 10), (100, 200)], 5)
    row = 12 * 128
    x = [synth.uniform_bf16(7 + i, 1, (c.N, row), -2, 2) for i in range(3)]
    src, qkv = empty((c.N, row), np.uint16), empty((c.N, row), np.uint16)
    pos_in, pos = empty(c.B, np.int32), empty(c.B, np.int32)
    cs = empty((c.pps * 16, 64, 2), np.float32)
    fp.fp_op_rope_table(c.pps * 16, 128, 10000.0, ptr(cs))
    a = torch.randn(4096, 4096, device="cuda")
    t = torch.empty_like(a)
    t2 = torch.empty_like(a)
    cu, err = dev(c.cu), empty(1, np.int32)

    def buffers():
        return empty((c.N, 1024), np.uint16), empty((c.N, 256), np.uint16), empty((c.N, 256), np.uint16), empty((c.N, 1024), np.uint16)

    out, plain = buffers(), buffers()
    need = fp.fp_op_attention_chunk_workspace_bytes(c.B, 8, 2, 128, c.max_new)
    ws = empty(need + 256)
    s0, s1 = torch.cuda.Stream(), torch.cuda.Stream()

    def calls(bufs, at, stream):
        q, k, v, o = bufs
        fp.fp_op_rope_kv_chunk(ptr(qkv), row, c.N, c.B, 8, c.view, ptr(cu), ptr(at), ptr(cs), ptr(q), 1024, ptr(err), stream)
        fp.fp_op_kv_read(c.view, c.N, c.B, ptr(cu), ptr(at), ptr(k), ptr(v), 256, ptr(err), stream)
        fp.fp_op_attention_chunk(ptr(q), 1024, c.N, c.B, 8, c.view, ptr(cu), ptr(at), c.max_new, c.max_len, ptr(o),
                                 (ptr(ws) + 255) // 256 * 256, need, ptr(err), stream)

    def step():
        s1.wait_stream(s0)
        with torch.cuda.stream(s1):
            torch.mm(a, a, out=t2)
            torch.mm(a, a, out=t2)
            torch.add(pos_in, 0, out=pos)  # (a kernel, behind the products)
        with torch.cuda.stream(s0):
            torch.mm(a, a, out=t)
            torch.add(src, 0, out=qkv)
            s0.wait_stream(s1)
            calls(out, pos, s0.cuda_stream)

    torch.cuda.synchronize()
    with torch.cuda.stream(s0):  # (the library's own set-up, outside the capture)
        torch.mm(a, a, out=t)
        s1.wait_stream(s0)
    with torch.cuda.stream(s1):
        torch.mm(a, a, out=t2)
    torch.cuda.synchronize()
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s0):
            step()
    base = {w: v.clone() for w, v in c.dev.items()}
    for turn in range(3):
        where = np.array([10 + turn, 200 - turn], np.int32)
        for w in base:
            c.dev[w].copy_(base[w])
        src.copy_(torch.from_numpy(x[turn].view(np.int16)))
        pos_in.copy_(torch.from_numpy(where))
        qkv.zero_()
        pos.zero_()
        for o in out:
            o.zero_()
        torch.cuda.synchronize()
        if graph:
            g.replay()
        else:
            step()
        torch.cuda.synchronize()
        assert host(err, np.int32)[0] == 0
        got = [host(o, np.uint16).copy() for o in out]
        for w in base:
            c.dev[w].copy_(base[w])
        torch.cuda.synchronize()
        calls(plain, dev(where), None)
        torch.cuda.synchronize()
        for o, p in zip(got, plain):
            assert np.array_equal(o, host(p, np.uint16)), turn
        assert np.array_equal(host(qkv, np.uint16).reshape(x[turn].shape), x[turn])
