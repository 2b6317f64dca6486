"""Refusals of the tree and beam operators, decided on the host before any CUDA call: these run without a GPU."""
import os
import re

import pytest

from tests.test_chunk_abi import A, CAPACITY, INVALID, UNSUPPORTED, code, fp, view  # noqa: F401


def test_tree_plan_refusals(fp):  # noqa: F811
    def call(parent=A, n=4, B=2, cu=A, most=8, depth=A, mask=A, stride=1):
        return code(lambda: fp.fp_op_tree_plan(parent, n, B, cu, most, depth, mask, stride))

    for kw in (dict(parent=None), dict(n=-1), dict(B=-1), dict(cu=None), dict(most=-1), dict(depth=None), dict(mask=None),
               dict(stride=0), dict(most=33), dict(most=1024, stride=31)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(most=1025, stride=33), dict(stride=(1 << 16) + 1), dict(n=(1 << 30) + 1), dict(B=(1 << 26) + 1)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(n=0) == 0 and call(B=0) == 0 and call(most=0, stride=0) == 0


def test_rope_kv_tree_refusals(fp):  # noqa: F811
    def call(kv=None, qkv=A, row=1024, n=4, B=2, H=4, cu=A, pos=A, depth=A, cs=A, q=2 * A, qs=512, **kw):
        return code(lambda: fp.fp_op_rope_kv_tree(qkv, row, n, B, H, kv or view(fp, **kw), cu, pos, depth, cs, q, qs))

    for kw in (dict(qkv=None), dict(cu=None), dict(pos=None), dict(cs=None), dict(q=None), dict(n=-1), dict(B=-1),
               dict(H=3), dict(H=0), dict(row=1016), dict(qs=504), dict(kvq=2), dict(kvq=1), dict(k=None),
               dict(table=None), dict(Hkv=0), dict(q=A), dict(depth=None)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(qkv=A + 8), dict(q=A + 2), dict(cs=A + 4), dict(row=1028), dict(qs=516), dict(hd=96), dict(page=32),
               dict(k=A + 8), dict(v=A + 8), dict(pages=1 << 26)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(n=0) == 0 and call(B=0) == 0


def test_attention_tree_refusals(fp):  # noqa: F811
    need = fp.fp_op_attention_tree_workspace_bytes(2, 4, 2, 128, 8)
    assert need > 0

    def call(q=A, qs=512, n=4, B=2, H=4, cu=A, pos=A, mask=A, stride=1, max_new=8, max_len=64, out=A, ws=A, wsb=need, **kw):
        return code(lambda: fp.fp_op_attention_tree(q, qs, n, B, H, view(fp, **kw), cu, pos, mask, stride, max_new, max_len,
                                                    out, ws, wsb))

    for kw in (dict(q=None), dict(cu=None), dict(pos=None), dict(out=None), dict(n=-1), dict(B=-1), dict(H=3),
               dict(H=0), dict(qs=504), dict(max_new=-1), dict(max_len=-1), dict(ws=None), dict(wsb=need - 1),
               dict(ws=A + 128), dict(kvq=1), dict(k=None), dict(mask=None), dict(stride=0), dict(max_new=33)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(q=A + 8), dict(out=A + 8), dict(qs=516), dict(hd=96), dict(page=8), dict(v=A + 4),
               dict(H=258, qs=258 * 128), dict(pages=1 << 26), dict(n=(1 << 30) + 1),
               dict(B=(1 << 26) + 1), dict(pps=1 << 26, max_len=1 << 30, n=1 << 28)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(max_len=65) == CAPACITY
    assert call(n=0) == 0 and call(B=0) == 0 and call(max_new=0) == 0 and call(max_len=0) == 0


def test_attention_tree_workspace_query(fp):  # noqa: F811
    f = fp.fp_op_attention_tree_workspace_bytes
    assert f(0, 4, 2, 128, 8) == f(2, 0, 2, 128, 8) == f(2, 4, 0, 128, 8) == f(2, 4, 2, 128, 0) == 0
    assert f(2, 4, 2, 96, 8) == f(2, 5, 2, 128, 8) == f(2, 258, 2, 128, 8) == 0
    assert 0 < f(1, 8, 8, 64, 1) <= f(1000, 64, 8, 128, 4096) < 1 << 28


def test_verify_tree_refusals(fp):  # noqa: F811
    def call(p=A, V=5, n=4, B=2, cu=A, parent=A, tok=A, u=A, path=A, out=A, cnt=A):
        return code(lambda: fp.fp_op_verify_tree(p, V, n, B, cu, parent, tok, u, path, out, cnt))

    for kw in (dict(p=None), dict(V=0), dict(n=-1), dict(B=-1), dict(cu=None), dict(parent=None), dict(tok=None),
               dict(u=None), dict(path=None), dict(out=None), dict(cnt=None)):
        assert call(**kw) == INVALID, kw
    assert call(V=(1 << 30) + 1) == call(B=(1 << 27) + 1) == UNSUPPORTED
    assert call(B=0) == 0


def test_kv_commit_refusals(fp):  # noqa: F811
    call = lambda n=4, B=2, cu=A, pos=A, path=A, **kw: code(  # noqa: E731
        lambda: fp.fp_op_kv_commit(view(fp, **kw), n, B, cu, pos, path))
    for kw in (dict(n=-1), dict(B=-1), dict(cu=None), dict(pos=None), dict(path=None), dict(kvq=1), dict(kvq=3), dict(Hkv=0)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(hd=32), dict(k=A + 2), dict(page=8), dict(pages=1 << 26), dict(B=(1 << 26) + 1)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(n=0) == 0 and call(B=0) == 0


def test_beam_select_refusals(fp):  # noqa: F811
    need = fp.fp_op_beam_select_workspace_bytes(2, 4, 5)
    assert need > 0

    def call(x=A, V=5, B=2, W=4, score=A, done=A, end=2, parent=A, token=A, out=A, nd=A, ws=A, wsb=need):
        return code(lambda: fp.fp_op_beam_select(x, V, B, W, score, done, end, parent, token, out, nd, ws, wsb))

    for kw in (dict(x=None), dict(V=0), dict(B=-1), dict(W=0), dict(W=-2), dict(score=None), dict(end=-2), dict(end=5),
               dict(end=-1), dict(parent=None), dict(token=None), dict(out=None), dict(ws=None), dict(ws=A + 128),
               dict(wsb=need - 1)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(W=33), dict(B=16385), dict(V=(1 << 30) + 1)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(B=0) == 0
    f = fp.fp_op_beam_select_workspace_bytes
    assert f(0, 4, 5) == f(2, 0, 5) == f(2, 33, 5) == f(2, 4, 0) == f(16385, 4, 5) == f(2, 4, (1 << 30) + 1) == 0
    assert 0 < f(1, 1, 1) < f(64, 32, 200000) < 1 << 30


def test_beam_reorder_refusals(fp):  # noqa: F811
    def call(B=2, W=4, pps=3, page=16, n=A, parent=A, tin=A, tout=2 * A, src=A, dst=A, rows=A):
        return code(lambda: fp.fp_op_beam_reorder(B, W, pps, page, n, parent, tin, tout, src, dst, rows))

    for kw in (dict(B=-1), dict(W=0), dict(pps=0), dict(page=0), dict(n=None), dict(parent=None), dict(tin=None),
               dict(tout=None), dict(tout=A), dict(src=None), dict(dst=None), dict(rows=None)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(W=33), dict(B=16385), dict(page=32), dict(pps=(1 << 26) + 1)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(B=0) == 0


def test_kv_copy_refusals(fp):  # noqa: F811
    call = lambda n=4, src=A, dst=A, rows=A, **kw: code(lambda: fp.fp_op_kv_copy(view(fp, **kw), n, src, dst, rows))  # noqa: E731
    for kw in (dict(n=-1), dict(src=None), dict(dst=None), dict(rows=None), dict(kvq=1), dict(kvq=3), dict(k=None)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(hd=32), dict(k=A + 2), dict(v=A + 8), dict(page=8)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(n=0) == 0


def test_headers_declare_the_binding_arguments(fp):  # noqa: F811
    """The C prototypes take as many arguments as the binding passes, and the limits agree."""
    src = open(os.path.join(os.path.dirname(__file__), "..", "include", "fp_ops.h")).read()
    for name in ("FP_TREE_MAX_ROWS", "FP_BEAM_MAX", "FP_BEAM_MAX_GROUPS"):
        assert int(re.search(r"#define %s (\d+)" % name, src).group(1)) == getattr(fp, name)
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    for name in ("fp_op_tree_plan", "fp_op_rope_kv_tree", "fp_op_attention_tree", "fp_op_attention_tree_workspace_bytes",
                 "fp_op_verify_tree", "fp_op_kv_commit", "fp_op_beam_select", "fp_op_beam_select_workspace_bytes",
                 "fp_op_beam_reorder", "fp_op_kv_copy"):
        args = re.search(r"\b%s\s*\(([^)]*)\)" % name, src).group(1)
        assert len(args.split(",")) == len(getattr(fp._lib, name).argtypes), name
        assert callable(getattr(fp, name))
