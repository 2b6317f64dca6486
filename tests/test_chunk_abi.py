"""Refusals of the chunk operators, decided on the host before any CUDA call: these run without a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def fp():
    import __graft_entry__

    __graft_entry__.build()
    import paper_2501_13111_gb300 as fp

    return fp


INVALID, UNSUPPORTED, CAPACITY = -1, -2, -5
A = 4096  # any aligned address: nothing is launched


def view(fp, kvq=0, Hkv=2, hd=128, page=16, pps=4, pages=8, k=A, v=A, ks=None, vs=None, table=A):
    return fp.fp_kv_view(kvq, Hkv, hd, page, pps, pages, k, v, ks, vs, table)


def code(call):
    try:
        call()
    except Exception as e:
        return e.code
    return 0


def test_rope_kv_chunk_refusals(fp):
    def call(kv=None, qkv=A, row=1024, n=4, B=2, H=4, cu=A, pos=A, cs=A, q=2 * A, qs=512, **kw):
        return code(lambda: fp.fp_op_rope_kv_chunk(qkv, row, n, B, H, kv or view(fp, **kw), cu, pos, cs, q, qs))

    for kw in (dict(qkv=None), dict(cu=None), dict(pos=None), dict(cs=None), dict(q=None), dict(n=-1), dict(B=-1),
               dict(H=3), dict(H=0), dict(row=1016), dict(qs=504), dict(kvq=2), dict(kvq=1), dict(k=None),
               dict(table=None), dict(Hkv=0), dict(q=A)):
        assert call(**kw) == INVALID, kw
    assert call(q=A, qs=1024, n=0) == 0
    for kw in (dict(qkv=A + 8), dict(q=A + 2), dict(cs=A + 4), dict(row=1028), dict(qs=516), dict(hd=96), dict(page=32),
               dict(k=A + 8), dict(v=A + 8), dict(pages=1 << 26)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(n=0) == 0 and call(B=0) == 0


def test_kv_read_refusals(fp):
    def call(n=4, B=2, cu=A, pos=A, k_out=A, v_out=A, stride=256, **kw):
        return code(lambda: fp.fp_op_kv_read(view(fp, **kw), n, B, cu, pos, k_out, v_out, stride))

    for kw in (dict(cu=None), dict(pos=None), dict(k_out=None), dict(v_out=None), dict(n=-1), dict(B=-1),
               dict(stride=248), dict(kvq=1), dict(kvq=3)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(k_out=A + 8), dict(v_out=A + 8), dict(stride=260), dict(hd=32), dict(k=A + 2)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(n=0) == 0 and call(B=0) == 0


def test_attention_chunk_refusals(fp):
    need = fp.fp_op_attention_chunk_workspace_bytes(2, 4, 2, 128, 8)
    assert need > 0

    def call(q=A, qs=512, n=4, B=2, H=4, cu=A, pos=A, max_new=8, max_len=64, out=A, ws=A, wsb=need, **kw):
        return code(lambda: fp.fp_op_attention_chunk(q, qs, n, B, H, view(fp, **kw), cu, pos, max_new, max_len, out, ws,
                                                     wsb))

    for kw in (dict(q=None), dict(cu=None), dict(pos=None), dict(out=None), dict(n=-1), dict(B=-1), dict(H=3),
               dict(H=0), dict(qs=504), dict(max_new=-1), dict(max_len=-1), dict(ws=None), dict(wsb=need - 1),
               dict(ws=A + 128), dict(kvq=1), dict(k=None)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(q=A + 8), dict(out=A + 8), dict(qs=516), dict(hd=96), dict(page=8), dict(v=A + 4),
               dict(H=258, qs=258 * 128), dict(pages=1 << 26), dict(n=(1 << 30) + 1),
               dict(B=(1 << 26) + 1), dict(pps=1 << 26, max_len=1 << 30, n=1 << 28)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(max_len=65) == CAPACITY
    assert call(n=0) == 0 and call(B=0) == 0 and call(max_new=0) == 0 and call(max_len=0) == 0


def test_attention_chunk_workspace_query(fp):
    f = fp.fp_op_attention_chunk_workspace_bytes
    assert f(0, 4, 2, 128, 8) == f(2, 0, 2, 128, 8) == f(2, 4, 0, 128, 8) == f(2, 4, 2, 128, 0) == 0
    assert f(2, 4, 2, 96, 8) == f(2, 5, 2, 128, 8) == f(2, 258, 2, 128, 8) == 0
    assert 0 < f(1, 8, 8, 64, 1) <= f(1000, 64, 8, 128, 4096) < 1 << 28


def test_softmax_refusals(fp):
    call = lambda x=A, M=2, V=5, t=None, y=A: code(lambda: fp.fp_op_softmax(x, M, V, t, y))  # noqa: E731
    for kw in (dict(x=None), dict(y=None), dict(M=-1), dict(V=0), dict(V=-3)):
        assert call(**kw) == INVALID, kw
    assert call(M=(1 << 27) + 1) == call(V=(1 << 30) + 1) == UNSUPPORTED
    assert call(M=0) == 0


def test_verify_draft_refusals(fp):
    def call(p=A, q=A, V=5, n=4, B=2, cu=A, tok=A, u=A, r=A, out=A, cnt=A):
        return code(lambda: fp.fp_op_verify_draft(p, q, V, n, B, cu, tok, u, r, out, cnt))

    for kw in (dict(p=None), dict(V=0), dict(n=-1), dict(B=-1), dict(cu=None), dict(tok=None), dict(u=None),
               dict(r=None), dict(out=None), dict(cnt=None)):
        assert call(**kw) == INVALID, kw
    assert call(V=(1 << 30) + 1) == UNSUPPORTED
    assert call(B=0) == 0


def test_headers_declare_the_binding_arguments(fp):
    """The C prototypes take as many arguments as the binding passes."""
    import os
    import re

    src = open(os.path.join(os.path.dirname(__file__), "..", "include", "fp_ops.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    for name in ("fp_op_rope_kv_chunk", "fp_op_kv_read", "fp_op_attention_chunk", "fp_op_softmax", "fp_op_verify_draft",
                 "fp_op_attention_chunk_workspace_bytes"):
        args = re.search(r"\b%s\s*\(([^)]*)\)" % name, src).group(1)
        assert len(args.split(",")) == len(getattr(fp._lib, name).argtypes), name
        assert isinstance(getattr(fp, name), type(code)) and C is not None
