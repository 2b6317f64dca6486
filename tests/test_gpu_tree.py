"""Trees of drafted tokens against the oracle: plan, append, attention, verification, commit, and a whole step.

The attention's tolerance is that of the chunk's (tests/test_gpu_chunk.py):
    |got - o| <= 2^-8 |o| + (2^-8 + 2^-10) sum_j p_j |v_j|.
Plans, accepted paths, drawn tokens and committed rows are exact.
"""
import numpy as np
import pytest

import synth
from oracle import model as M
from oracle import quant, several
from tests.gpu_helpers import dev, empty, host, ptr, torch_mod
from tests.test_gpu_chunk import BASE, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def grow(rng, n, how):
    """Parents of n rows: a chain, a star, or at random."""
    if how == "chain":
        return [i - 1 for i in range(n)]
    if how == "star":
        return [-1, *[0] * (n - 1)][:n]
    return [-1, *[int(rng.integers(0, i)) for i in range(1, n)]][:n]


class Trees(Batch):
    """A Batch whose sequences' rows are trees."""

    def __init__(self, fp, kvq, hd, H, Hkv, seqs, seed, how="random", words=None, **kw):
        super().__init__(fp, kvq, hd, H, Hkv, seqs, seed, **kw)
        rng = np.random.default_rng(seed + 1000)
        self.parents = [grow(rng, n, how) for n, _ in seqs]
        self.seen = [several.plan(p)[1] for p in self.parents]
        self.words = words or (self.max_new + 31) // 32
        self.mask = np.full((self.N, self.words), 0xFFFFFFFF, np.uint32)
        for b, s in enumerate(self.seen):
            self.mask[self.cu[b] : self.cu[b] + len(s)] = several.words(s, self.words)

    def flat(self, lists, fill=-1):
        out = np.full(self.N, fill, np.int32)
        for b, x in enumerate(lists):
            out[self.cu[b] : self.cu[b] + len(x)] = x
        return out

    def attend(self, q, out=None, cu=None, pos=None, mask=None, max_new=None, max_len=None, ws=None, stream=None, sync=True, view=None):
        f = self.fp
        qd = q if hasattr(q, "data_ptr") else dev(q)
        out = out if out is not None else dev(np.full((self.N, self.H * self.hd), 0x4321, np.uint16))
        need = f.fp_op_attention_tree_workspace_bytes(self.B, self.H, self.Hkv, self.hd, max_new or self.max_new)
        if ws is None:
            ws = empty(need + 256)
            ws[65536:] = 255
        err = empty(1, np.int32)
        m = self.mask if mask is None else mask
        f.fp_op_attention_tree(ptr(qd), qd.shape[1], self.N, self.B, self.H, view or self.view,
                               ptr(dev(self.cu if cu is None else cu)), ptr(dev(self.pos if pos is None else pos)),
                               ptr(dev(m)), m.shape[1], max_new or self.max_new, max_len or self.max_len, ptr(out),
                               (ptr(ws) + 255) // 256 * 256, need, ptr(err), stream)
        if not sync:
            return out, err
        return host(out, np.uint16).reshape(self.N, self.H * self.hd), int(host(err, np.int32)[0])

    def visible(self, b, seen=None):
        n, p = self.seqs[b]
        v = np.zeros((n, p + n), bool)
        v[:, :p] = True
        for i, s in enumerate((seen or self.seen)[b]):
            v[i, [p + j for j in s if j < n]] = True
        return v

    def check(self, q, got, only=None, seen=None):
        H, hd = self.H, self.hd
        owned = np.zeros(self.N, bool)
        for b, (n, p) in enumerate(self.seqs):
            r = slice(int(self.cu[b]), int(self.cu[b]) + n)
            owned[r] = True
            if n == 0 or (only is not None and b not in only):
                continue
            k, v = self.cached("k", b, p + n), self.cached("v", b, p + n)
            x = quant.bf16_to_f32(q[r, : H * hd]).astype(np.float64).reshape(n, H, hd)
            o = quant.bf16_to_f32(got[r]).astype(np.float64).reshape(n, H, hd)
            vis = self.visible(b, seen)
            ref, mass = several.attention(x, vis, k, v), several.attention(x, vis, k, np.abs(v))
            off = np.abs(o - ref) / (2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * mass + 1e-30)
            assert np.all(np.isfinite(o)) and off.max() <= 1, (b, off.max(), np.argwhere(off == off.max())[:3])
        assert np.all(got[~owned] == 0x4321)


# ------------------------------------------------------------------ plan
def run_plan(fp, parents, cu, N, most, stride, B=None):
    depth, mask = dev(np.full(N, 77, np.int32)), dev(np.full((N, stride), 0x5A5A5A5A, np.uint32))
    err = empty(1, np.int32)
    fp.fp_op_tree_plan(ptr(dev(parents)), N, B or len(cu) - 1, ptr(dev(np.array(cu, np.int32))), most, ptr(depth), ptr(mask),
                       stride, ptr(err))
    return host(depth, np.int32), host(mask, np.uint32).reshape(N, stride), int(host(err, np.int32)[0])


@pytest.mark.parametrize("how", ["random", "chain", "star"])
@pytest.mark.parametrize("ns,extra", [([1], 0), ([5, 0, 32, 33, 1, 31, 64], 0), ([1024], 0), ([300, 7], 2), ([1000, 1023, 2], 1)])
def test_plan(fp, ns, extra, how):
    rng = np.random.default_rng(sum(ns))
    trees = [grow(rng, n, how) for n in ns]
    cu = 2 + np.concatenate([[0], np.cumsum(ns)])
    N = int(cu[-1]) + 3
    flat = np.full(N, 99, np.int32)
    for b, t in enumerate(trees):
        flat[cu[b] : cu[b + 1]] = t
    stride = (max(ns) + 31) // 32 + extra
    depth, mask, err = run_plan(fp, flat, cu, N, max(ns), stride)
    assert err == 0
    owned = np.zeros(N, bool)
    for b, t in enumerate(trees):
        d, seen, _ = several.plan(t)
        owned[cu[b] : cu[b + 1]] = True
        assert depth[cu[b] : cu[b + 1]].tolist() == d
        assert np.array_equal(mask[cu[b] : cu[b + 1]], several.words(seen, stride))
    assert np.all(depth[~owned] == 77) and np.all(mask[~owned] == 0x5A5A5A5A)


def test_plan_reports_impossible_parents_and_too_many_rows(fp):
    flat = np.array([-1, 0, 1, 3, -2, 4, 2 ** 31 - 1, -2 ** 31, 0], np.int32)
    depth, mask, err = run_plan(fp, flat, [0, 9], 9, 9, 1)
    assert err == 1 and depth.tolist() == several.plan(flat.tolist())[0]
    assert np.array_equal(mask, several.words(several.plan(flat.tolist())[1], 1))
    depth, mask, err = run_plan(fp, np.array([-1, 0, 1, 2, 3], np.int32), [0, 5], 5, 3, 1)
    assert err == 1 and depth.tolist() == [0, 1, 2, 77, 77] and mask[:, 0].tolist() == [1, 3, 7, 0x5A5A5A5A, 0x5A5A5A5A]
    for cu in ([0, 4, 2, 9], [0, 3, 6, 12], [-4, 3, 5, 9]):
        assert run_plan(fp, np.zeros(9, np.int32) - 1, cu, 9, 9, 1)[2] == 1
    assert run_plan(fp, np.zeros(9, np.int32) - 1, [0, 0, 0], 9, 9, 1)[2] == 0


# ------------------------------------------------------------------ attention
HEADS = [(64, 8, 8), (128, 8, 1), (128, 64, 8), (128, 6, 2), (64, 14, 2), (128, 5, 5), (128, 40, 2), (64, 128, 1)]
BATCHES = [
    [(1, 0)],
    [(3, 0), (0, 17), (1, 300), (5, 15), (130, 1), (16, 112)],
    [(1, 126), (2, 126), (3, 127), (2, 128), (1, 128), (17, 240)],
    [(260, 511)],
    [(16, 1000), (1, 3), (33, 257), (64, 900)] * 5,
    [(4, 5000)],
]


@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("hd,H,Hkv", HEADS)
@pytest.mark.parametrize("kvq", [0, 1])
def test_attention(fp, kvq, hd, H, Hkv, batch):
    c = Trees(fp, kvq, hd, H, Hkv, BATCHES[batch], 7 * batch + hd + H, lead=batch % 2 * 3, tail=5)
    q = c.queries(batch)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("kvq,hd,H,Hkv,seqs", [
    (0, 128, 8, 1, [(300, 1300), (1, 1999), (33, 64)]),
    (1, 128, 16, 2, [(513, 1023), (128, 0), (129, 127)]),
    (0, 64, 4, 4, [(1024, 0), (2, 700)]),
    (0, 128, 8, 1, [(64, 30000)]),
    (1, 128, 8, 1, [(1, 20000), (20, 7)]),
    (1, 64, 3, 1, [(100, 9000)]),
])
def test_attention_large_trees_and_units_that_many_ctas_share(fp, kvq, hd, H, Hkv, seqs):
    c = Trees(fp, kvq, hd, H, Hkv, seqs, 61, words=(max(n for n, _ in seqs) + 31) // 32 + 2)
    q = c.queries(14)
    ws = empty(fp.fp_op_attention_tree_workspace_bytes(c.B, H, Hkv, hd, c.max_new) + 256)
    for _ in range(2):
        got, err = c.attend(q, ws=ws)
        assert err == 0
        c.check(q, got)
    off = -ptr(ws) % 256
    assert not host(ws, np.uint8)[off:off + 65536].any()


@pytest.mark.parametrize("kvq,hd,H,Hkv,B", [(0, 128, 8, 2, 33), (1, 128, 8, 2, 75), (1, 64, 4, 4, 1100), (0, 64, 4, 1, 1100)])
def test_attention_of_many_sequences(fp, kvq, hd, H, Hkv, B):
    """More sequences than a warp has lanes, and than the GPU has SMs; some without rows."""
    rng = np.random.default_rng(B)
    c = Trees(fp, kvq, hd, H, Hkv, [(int(rng.integers(0, 6)), int(rng.integers(0, 200))) for _ in range(B)], B)
    q = c.queries(3)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_whatever_rows_are_announced(fp, hd):
    """An int8 cache, trees of one query tile: the same rows whether the bound on a tree's rows is one tile or many."""
    c = Trees(fp, 1, hd, 16, 2, [(16, 2000), (3, 40), (0, 5), (9, 700)], 9, words=32)
    q = c.queries(4)
    for most in (16, 17, 1024):
        got, err = c.attend(q, max_new=most)
        assert err == 0
        c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_any_mask(fp, kvq):
    """Masks that no tree has: rows that see later rows, none of their own, all; bits behind the rows do not count."""
    seqs = [(40, 0), (7, 100), (70, 250), (1, 0), (128, 31)]
    c = Trees(fp, kvq, 128, 8, 2, seqs, 5)
    rng = np.random.default_rng(3)
    c.mask = rng.integers(0, 1 << 32, c.mask.shape, dtype=np.uint32)
    c.mask[::5] = 0
    c.mask[3::5] = 0xFFFFFFFF
    seen = [[{j for j in range(n) if c.mask[c.cu[b] + i, j // 32] >> np.uint32(j % 32) & 1} for i in range(n)]
            for b, (n, _) in enumerate(seqs)]
    q = c.queries(6)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got, seen=seen)
    assert not np.any(got[0:40:5] & 0x7FFF)  # rows that see nothing


@pytest.mark.parametrize("kvq", [0, 1])
@pytest.mark.parametrize("junk", [np.nan, np.inf, -3e38])
def test_attention_ignores_what_lies_behind_a_sequence(fp, kvq, junk):
    c = Trees(fp, kvq, 128, 8, 2, [(3, 10), (16, 0), (20, 250), (1, 127)], 11, junk=junk)
    q = c.queries(2)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_a_key_that_is_nan_reaches_the_rows_that_see_it(fp, kvq):
    """A drafted row's key of NaN (an int8 cache: its scale): its descendants are NaN, other branches keep their bits."""
    c = Trees(fp, kvq, 128, 8, 2, [(30, 100), (64, 300), (5, 2)], 13)
    q = c.queries(2)
    clean, err = c.attend(q)
    assert err == 0
    bad = np.zeros(c.N, bool)
    for b, (n, p) in enumerate(c.seqs):
        t = p + n // 3
        page, slot = int(c.table[b, t // 16]), t % 16
        if kvq:
            c.dev["ks"][page, :, slot] = float("nan")
        else:
            c.dev["k"].view(torch_mod().bfloat16)[page, :, slot, 5] = float("nan")
        for i, s in enumerate(c.seen[b]):
            bad[c.cu[b] + i] = n // 3 in s
    got, err = c.attend(q)
    assert err == 0 and bad.any() and not bad.all()
    assert np.all(np.isnan(quant.bf16_to_f32(got[bad])))
    assert np.array_equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_of_chains_is_the_chunk_s(fp, kvq):
    """Chains see what a chunk's rows see; the same masks either way, so the same tolerance holds."""
    c = Trees(fp, kvq, 128, 16, 2, [(5, 700), (1, 90), (40, 33)], 17, how="chain")
    q = c.queries(3)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)
    Batch.check(c, q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_beyond_the_bounds(fp, kvq):
    """Negative positions: no keys; behind max_len: not read; behind max_new: left; all reported."""
    c = Trees(fp, kvq, 128, 8, 2, [(6, 0), (9, 60), (40, 30)], 29)
    q = c.queries(9)
    got, err = c.attend(q, pos=np.array([-3, 60, 30], np.int32))
    assert err == 1 and not np.any(got[:6] & 0x7FFF)
    c.check(q, got, only={1, 2})
    got, err = c.attend(q, max_len=66)  # sequence 1 ends at 69, 2 at 70
    assert err == 1
    seen = [c.seen[0], [{j for j in s if j < 6} for s in c.seen[1]], [{j for j in s if j < 36} for s in c.seen[2]]]
    c.check(q, got, seen=seen)
    got, err = c.attend(q, max_new=4)
    assert err == 1
    assert np.all(got[4:6] == 0x4321) and np.all(got[10:15] == 0x4321) and np.all(got[19:] == 0x4321)
    x = np.array(got)
    x[4:6] = 0
    for cu in ([0, 6, 15, 90], [-3, 6, 15, 55], [0, 15, 6, 55], [100, 200, 300, 400]):
        got, err = c.attend(q, cu=np.array(cu, np.int32))
        assert err == 1 and np.all(got == 0x4321), cu


def test_attention_bad_page_reads_zeros(fp):
    for kvq in (0, 1):
        c = Trees(fp, kvq, 128, 8, 2, [(6, 100), (4, 40)], 31)
        q = c.queries(9)
        table = c.table.copy()
        table[0, 2], table[1, 0] = c.pages, -1
        got, err = c.attend(q, view=c.make_view(table))
        assert err == 1
        whole = c.cached
        c.cached = lambda w, b, length: whole(w, b, length, table)
        c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_captured_and_replayed_with_other_trees(fp, kvq):
    """One captured launch within bounds serves other batches and masks; two graphs share a workspace in turn."""
    torch = torch_mod()
    a = Trees(fp, kvq, 128, 16, 2, [(5, 700), (1, 90), (3, 33)], 37, tail=60, words=2)
    q = a.queries(12)
    qd, out = dev(q), dev(np.full((a.N, a.H * a.hd), 0x4321, np.uint16))
    cu, pos, mask, err = dev(a.cu), dev(a.pos), dev(a.mask), empty(1, np.int32)
    need = fp.fp_op_attention_tree_workspace_bytes(a.B, a.H, a.Hkv, a.hd, 40)
    ws = empty(need + 256)
    st = torch.cuda.Stream()

    def call():
        fp.fp_op_attention_tree(ptr(qd), qd.shape[1], a.N, a.B, a.H, a.view, ptr(cu), ptr(pos), ptr(mask), 2, 40, a.max_len,
                                ptr(out), (ptr(ws) + 255) // 256 * 256, need, ptr(err), st.cuda_stream)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            call()
        graphs.append(g)
    rng = np.random.default_rng(5)
    for turn, seqs in enumerate([[(5, 700), (1, 90), (3, 33)], [(1, 0), (40, 660), (0, 9)], [(2, 5), (2, 6), (40, 300)]]):
        a.seqs = seqs
        a.cu = np.concatenate([[0], np.cumsum([s[0] for s in seqs])]).astype(np.int32)
        a.seen = [several.plan(grow(rng, n, "random"))[1] if n else [] for n, _ in seqs]
        m = np.zeros((a.N, 2), np.uint32)
        for b, s in enumerate(a.seen):
            if s:
                m[a.cu[b] : a.cu[b + 1]] = several.words(s, 2)
        cu.copy_(torch.from_numpy(a.cu))
        pos.copy_(torch.from_numpy(np.array([s[1] for s in seqs], np.int32)))
        mask.copy_(torch.from_numpy(m.view(np.int32)))
        out.fill_(0x4321)
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        a.check(q, host(out, np.uint16).reshape(a.N, -1))
    assert host(err, np.int32)[0] == 0


def test_attention_repeats_bit_for_bit(fp):
    torch = torch_mod()
    c = Trees(fp, 1, 128, 64, 8, [(5, 2100), (30, 900), (64, 1200), (1, 4000)], 41)
    qd = dev(c.queries(13))
    first = c.attend(qd)[0]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [c.attend(qd, stream=s.cuda_stream, sync=False)[0] for s in streams]
    torch.cuda.synchronize()
    for o in outs:
        assert np.array_equal(host(o, np.uint16).reshape(first.shape), first)


@pytest.mark.parametrize("kvq", [0, 1])
def test_an_expired_wait_is_reported(fp, kvq):
    """The failure path, without a fault; after the tickets are zeroed again the workspace serves the same batch."""
    c = Trees(fp, kvq, 128, 64, 8, [(5, 700), (40, 900), (1, 2000), (3, 20)] * 3, 101)
    q = c.queries(6)
    ws = empty(fp.fp_op_attention_tree_workspace_bytes(c.B, c.H, c.Hkv, c.hd, c.max_new) + 256)
    fp.fp_debug_set_wait_limit(0)
    try:
        _, err = c.attend(q, ws=ws)
    finally:
        fp.fp_debug_set_wait_limit(-1)
    assert err == 2
    at = -ptr(ws) % 256
    ws[at:at + 65536] = 0
    got, err = c.attend(q, ws=ws)
    assert err == 0
    c.check(q, got)


# ------------------------------------------------------------------ append
def _table(fp, pps, hd):
    cs = empty((pps * 16, hd // 2, 2), np.float32)
    fp.fp_op_rope_table(pps * 16, hd, BASE, ptr(cs))
    return cs


def _append(c, qkv, depth, pos=None, view=None):
    f = c.fp
    out = {"q": dev(np.full((c.N, c.H * c.hd), 0x4321, np.uint16))}
    for w in "kv":
        out[w] = dev(np.full((c.N, c.Hkv * c.hd), 0x4321, np.uint16))
    err = empty(1, np.int32)
    args = ptr(dev(c.cu)), ptr(dev(c.pos if pos is None else pos))
    f.fp_op_rope_kv_tree(ptr(dev(qkv)), qkv.shape[1], c.N, c.B, c.H, view or c.view, *args, ptr(dev(depth)),
                         ptr(_table(f, c.pps, c.hd)), ptr(out["q"]), c.H * c.hd, ptr(err))
    e = int(host(err, np.int32)[0])
    f.fp_op_kv_read(view or c.view, c.N, c.B, *args, ptr(out["k"]), ptr(out["v"]), c.Hkv * c.hd, None)
    return {w: host(x, np.uint16).reshape(c.N, -1) for w, x in out.items()}, e


@pytest.mark.parametrize("hd,H,Hkv", [(64, 8, 8), (128, 8, 1), (128, 64, 8), (64, 6, 2)])
@pytest.mark.parametrize("kvq", [0, 1])
def test_append_rotates_by_depth_and_stores_by_row(fp, kvq, hd, H, Hkv):
    """Rotations against fp64: fp32 products and one bf16 rounding, 2^-8 of the value and 2^-22 of the pair; an int8 row
    then is off by half a step of its scale and, where the rounding to bf16 went the other way, a step of bf16, and the
    read back rounds once more.  Values bit for bit in a bf16 cache."""
    c = Trees(fp, kvq, hd, H, Hkv, [(6, 0), (33, 100), (0, 3), (1, 15), (16, 250)], 7, tail=2)
    qkv = synth.uniform_bf16(3, 1, (c.N, (H + 2 * Hkv) * hd), -2, 2)
    depth = c.flat([several.plan(p)[0] for p in c.parents], 0)
    got, err = _append(c, qkv, depth)
    assert err == 0
    x = quant.bf16_to_f32(qkv).astype(np.float64).reshape(c.N, -1, hd)
    for b, (n, p) in enumerate(c.seqs):
        r = slice(int(c.cu[b]), int(c.cu[b]) + n)
        y = M.rope(x[r, : H + Hkv], p + depth[r], BASE)
        pair = np.hypot(*np.split(y, 2, -1))
        tol = 2.0 ** -8 * np.abs(y) + 2.0 ** -21 * np.concatenate([pair, pair], -1)
        q = quant.bf16_to_f32(got["q"][r]).reshape(n, H, hd)
        assert np.all(np.abs(q - y[:, :H]) <= tol[:, :H])
        for w, ref, t in (("k", y[:, H:], tol[:, H:]), ("v", x[r, H + Hkv :], 0.0)):
            o = quant.bf16_to_f32(got[w][r]).reshape(n, Hkv, hd)
            if kvq:
                t = t + 0.51 * np.abs(ref).max(-1, keepdims=True) / 127 * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(o)
            assert np.all(np.abs(o - ref) <= t), (w, b)
    assert np.all(got["q"][-2:] == 0x4321)


@pytest.mark.parametrize("kvq", [0, 1])
def test_append_of_a_chain_is_the_chunk_s_bit_for_bit(fp, kvq):
    c = Trees(fp, kvq, 128, 8, 2, [(6, 10), (20, 100)], 9, how="chain")
    qkv = synth.uniform_bf16(4, 1, (c.N, 12 * 128), -2, 2)
    got, err = _append(c, qkv, c.flat([list(range(n)) for n, _ in c.seqs]))
    assert err == 0
    q, k, v = (empty((c.N, h * 128), np.uint16) for h in (8, 2, 2))
    args = ptr(dev(c.cu)), ptr(dev(c.pos))
    fp.fp_op_rope_kv_chunk(ptr(dev(qkv)), 12 * 128, c.N, c.B, 8, c.view, *args, ptr(_table(fp, c.pps, 128)), ptr(q), 1024)
    fp.fp_op_kv_read(c.view, c.N, c.B, *args, ptr(k), ptr(v), 256)
    for w, x in (("q", q), ("k", k), ("v", v)):
        assert np.array_equal(host(x, np.uint16).reshape(c.N, -1), got[w]), w


def test_append_skips_what_has_no_place(fp):
    c = Trees(fp, 0, 128, 4, 2, [(4, 10), (3, 20)], 11)
    qkv = synth.uniform_bf16(5, 1, (c.N, 8 * 128), -2, 2)
    before = {w: host(c.dev[w], np.uint16).copy() for w in "kv"}
    depth = c.flat([[0, 1, c.pps * 16, -11], [0, 1, 1]], 0)  # rotated outside the cache, behind and before
    got, err = _append(c, qkv, depth)
    assert err == 1
    assert np.all(got["q"][2:4] == 0x4321) and np.all(got["q"][[0, 1, 4, 5, 6]] != 0x4321)
    page = c.table[0, 0]
    for w in "kv":
        now = host(c.dev[w], np.uint16)
        assert np.array_equal(now[page, :, 12:14], before[w][page, :, 12:14])
        assert not np.array_equal(now[page, :, 10], before[w][page, :, 10])


# ------------------------------------------------------------------ commit
def _commit(c, paths, pos=None, view=None, cu=None, stream=None):
    err = empty(1, np.int32)
    c.fp.fp_op_kv_commit(view or c.view, c.N, c.B, ptr(dev(c.cu if cu is None else cu)),
                         ptr(dev(c.pos if pos is None else pos)), ptr(dev(c.flat(paths) if isinstance(paths, list) else paths)),
                         ptr(err), stream)
    e = int(host(err, np.int32)[0])
    return {w: host(t, c.data[w].dtype) for w, t in c.dev.items()}, e


def _committed(c, paths, table=None):
    out = {w: x.copy() for w, x in c.data.items()}
    t = c.table if table is None else table
    for b, path in enumerate(paths):
        p = c.seqs[b][1]
        for j, r in enumerate(path):
            a, z = t[b, (p + r) // 16], t[b, (p + j) // 16]
            if min(a, z) < 0 or max(a, z) >= c.pages:
                continue
            for w in out:
                out[w][z, :, (p + j) % 16] = out[w][a, :, (p + r) % 16]
    return out


@pytest.mark.parametrize("hd,Hkv", [(64, 1), (64, 9), (128, 8), (128, 3)])
@pytest.mark.parametrize("kvq", [0, 1])
def test_commit(fp, kvq, hd, Hkv):
    """Paths of one row to hundreds, dense and sparse, over page borders: all bits of the pools."""
    rng = np.random.default_rng(hd + Hkv)
    seqs = [(1, 5), (6, 13), (0, 4), (64, 30), (40, 0), (300, 77), (33, 15), (20, 100), (512, 3)]
    c = Trees(fp, kvq, hd, Hkv, Hkv, seqs, 19, lead=2, tail=3)
    paths = [[0], [0, 2, 3], [], sorted(rng.choice(64, 40, replace=False).tolist()), list(range(40)),
             list(range(1, 300)), [0] + list(range(2, 33)), [0, 7, 19], sorted(rng.choice(512, 200, replace=False).tolist())]
    got, err = _commit(c, paths)
    assert err == 0
    want = _committed(c, paths)
    for w in want:
        assert np.array_equal(got[w].reshape(want[w].shape).view(np.uint8), want[w].view(np.uint8)), w


@pytest.mark.parametrize("kvq", [0, 1])
def test_commit_reports_a_path_that_is_none(fp, kvq):
    """A path that does not ascend, or leaves the sequence, ends there; the others go on."""
    seqs = [(6, 10), (6, 40), (6, 0), (6, 20)]
    c = Trees(fp, kvq, 128, 4, 2, seqs, 21)
    flat = c.flat([[0, 2, 2, 4], [1, 3, 6, 5], [2, 4, -1, 5], [3, 4, 5]])
    got, err = _commit(c, flat)
    assert err == 1
    want = _committed(c, [[0, 2], [1, 3], [2, 4], [3, 4, 5]])
    for w in want:
        assert np.array_equal(got[w].reshape(want[w].shape).view(np.uint8), want[w].view(np.uint8)), w
    assert _commit(c, c.flat([[], [], [], []]))[1] == 0
    assert _commit(c, c.flat([[], [], [], [2 ** 31 - 1]]))[1] == 1


def test_commit_skips_what_has_no_place(fp):
    c = Trees(fp, 0, 128, 4, 2, [(20, 10), (20, 40)], 23)
    table = c.table.copy()
    table[0, 1] = -5
    paths = [[0, 3, 7, 18], [2, 3]]
    got, err = _commit(c, paths, view=c.make_view(table))
    assert err == 1
    want = _committed(c, paths, table)
    for w in want:
        assert np.array_equal(got[w].reshape(want[w].shape), want[w]), w
    c2 = Trees(fp, 0, 128, 4, 2, [(20, 10), (20, 40)], 23)
    got, err = _commit(c2, paths, pos=np.array([-30, 2 ** 31 - 1], np.int32))
    assert err == 1
    for w in c2.data:
        assert np.array_equal(got[w].reshape(c2.data[w].shape), c2.data[w])


# ------------------------------------------------------------------ verification
def _verify(fp, p, cu, parent, tokens, u, stream=None):
    N, V = p.shape
    B = len(cu) - 1
    path, out, cnt, err = dev(np.full(N, 55, np.int32)), dev(np.full(N, 55, np.int32)), dev(np.full(B, 55, np.int32)), empty(1, np.int32)
    fp.fp_op_verify_tree(ptr(dev(p)), V, N, B, ptr(dev(np.array(cu, np.int32))), ptr(dev(np.array(parent, np.int32))),
                         ptr(dev(np.array(tokens, np.int32))), ptr(dev(np.array(u, np.float32))), ptr(path), ptr(out),
                         ptr(cnt), ptr(err), stream)
    return host(path, np.int32), host(out, np.int32), host(cnt, np.int32), int(host(err, np.int32)[0])


def _expected(p, cu, parent, tokens, u):
    N = len(p)
    path, out, cnt, good = np.full(N, 55, np.int32), np.full(N, 55, np.int32), [], True
    for b in range(len(cu) - 1):
        r = slice(cu[b], cu[b + 1])
        if cu[b] == cu[b + 1]:
            cnt.append(0)
            continue
        a, o, ok = several.verify(p[r].astype(np.float64), parent[r], tokens[r], u[r])
        good &= ok
        path[r], out[r] = -1, -1
        path[cu[b] : cu[b] + len(a)] = a
        out[cu[b] : cu[b] + len(o)] = o
        cnt.append(len(o))
    return path, out, np.array(cnt, np.int32), int(not good)


def _same(got, want):
    for g, w in zip(got, want):
        assert np.array_equal(g, w), (g, w)


def _problem(seed, ns, V, lead=0, tail=0, hot=3):
    """Trees whose children carry the likely tokens of their parents, weights that do not add up to one."""
    rng = np.random.default_rng(seed)
    cu = (lead + np.concatenate([[0], np.cumsum(ns)])).astype(int)
    N = int(cu[-1]) + tail
    p = rng.random((N, V)).astype(np.float32) / V
    likely = rng.integers(0, V, (N, hot))
    for h in range(hot):
        p[np.arange(N), likely[:, h]] = 0.6 / (h + 1)
    parent, tokens = np.full(N, 9, np.int32), np.full(N, 123456, np.int32)
    for b, n in enumerate(ns):
        t = grow(rng, n, ("random", "chain", "star")[b % 3])
        parent[cu[b] : cu[b + 1]] = t
        for i in range(1, n):
            tokens[cu[b] + i] = likely[cu[b] + t[i], rng.integers(0, hot)]
    return p, cu, parent, tokens, rng.random(N).astype(np.float32)


@pytest.mark.parametrize("ns,V", [([1], 7), ([5, 0, 33, 1, 64], 1000), ([16] * 40, 517), ([60], 100003), ([8, 3], 32000),
                                  ([300], 130), ([2, 2, 2], 1), ([31], 4097)])
def test_verify(fp, ns, V):
    for seed in range(4):
        p, cu, parent, tokens, u = _problem(seed, ns, V, lead=seed % 2, tail=seed)
        _same(_verify(fp, p, cu, parent, tokens, u), _expected(p, cu, parent, tokens, u))


@pytest.mark.parametrize("ns,V", [([64] * 40, 517), ([300] * 7, 5003), ([1], 1 << 20), ([3], 300001), ([20, 21], 850001),
                                  ([7] * 30, 200003)])
def test_verify_every_way_of_drawing(fp, ns, V):
    """Thousands of rows (a warp each), rows of a million tokens (clusters, several groups a lane and chunk), and more
    than 2^25 weights in all (one row after the other)."""
    p, cu, parent, tokens, u = _problem(11, ns, V, lead=1, tail=2)
    _same(_verify(fp, p, cu, parent, tokens, u), _expected(p, cu, parent, tokens, u))


@pytest.mark.parametrize("n", [200, 1500])
def test_verify_goes_all_the_way_down(fp, n):
    """A chain whose every draft is certain; 1500 rows are more than are staged at once."""
    V = 300
    rng = np.random.default_rng(1)
    tokens = rng.integers(0, V, n)
    p = np.zeros((n, V), np.float32)
    p[np.arange(n - 1), tokens[1:]] = 0.25
    p[n - 1, 17] = 1.0
    got = _verify(fp, p, [0, n], np.arange(n) - 1, tokens, rng.random(n))
    assert got[0].tolist() == list(range(n)) and got[1].tolist() == tokens[1:].tolist() + [17] and got[2][0] == n and got[3] == 0


def test_verify_takes_the_lowest_of_equal_children(fp):
    """Two children with the drawn token: the lower row.  Roots beside row 0, and parents that are none, are never reached."""
    p = np.zeros((7, 4), np.float32)
    p[:, 2] = 1.0
    parent, tokens = [-1, -1, 0, 0, 5, 3, -7], [2, 2, 1, 2, 2, 2, 2]
    got = _verify(fp, p, [0, 7], parent, tokens, [0.5] * 7)
    assert got[0].tolist() == [0, 3, 5, -1, -1, -1, -1] and got[1].tolist() == [2, 2, 2, -1, -1, -1, -1] and got[2][0] == 3


@pytest.mark.parametrize("u", [0.0, 0.25, 0.5, 0.75, np.nextafter(np.float32(1), np.float32(0))])
def test_verify_draws_at_the_borders(fp, u):
    """Quarters that the sums hit exactly: the border itself belongs to the token behind it.  Unlikely tokens between."""
    p = np.zeros((1, 4000), np.float32)
    p[0, [5, 900, 901, 3999]] = 0.25
    got = _verify(fp, p, [0, 1], [-1], [0], [u])
    assert got[1][0] == [5, 900, 901, 3999][min(3, int(float(u) * 4))] and got[3] == 0


def test_verify_weighs_nan_and_negative_as_nothing(fp):
    p, cu, parent, tokens, u = _problem(3, [9, 5], 700)
    p[:, 100:300] = np.nan
    p[:, 300:350] = -1.0
    _same(_verify(fp, p, cu, parent, tokens, u), _expected(p, cu, parent, tokens, u))


def test_verify_of_no_rows(fp):
    """Sequences without rows, in a buffer that has some and in none at all; a cu that leaves the latter is reported."""
    p = np.ones((3, 5), np.float32)
    got = _verify(fp, p, [2, 2, 2], [-1] * 3, [0] * 3, [0.5] * 3)
    assert got[2].tolist() == [0, 0] and got[3] == 0 and np.all(got[0] == 55) and np.all(got[1] == 55)
    one = dev(np.zeros(4, np.float32))
    for cu, want in (([0, 0, 0], 0), ([0, 1, 0], 1)):
        cnt, err = dev(np.full(2, 55, np.int32)), empty(1, np.int32)
        fp.fp_op_verify_tree(ptr(one), 4, 0, 2, ptr(dev(np.array(cu, np.int32))), ptr(one), ptr(one), ptr(one), ptr(one), ptr(one),
                             ptr(cnt), ptr(err))
        assert host(cnt, np.int32).tolist() == [0, 0] and host(err, np.int32)[0] == want


def test_verify_reports_what_cannot_be_drawn(fp):
    """No weight, or an infinite one: the row is accepted, its token is none; the other sequences as ever."""
    p, cu, parent, tokens, u = _problem(5, [1, 6, 6], 300)
    p[0] = 0.0
    p[cu[1]] = np.inf
    want = _expected(p, cu, parent, tokens, u)
    assert want[3] == 1 and want[2][0] == 0 and want[2][1] == 0
    _same(_verify(fp, p, cu, parent, tokens, u), want)
    for bad in ([0, 5, 3, 13], [0, 9, 13, 14], [-2, 1, 7, 13]):
        assert _verify(fp, p, bad, parent, tokens, u)[3] == 1


def test_cache_offsets_past_32_bits(fp):
    """A pool of more than 2^32 elements: append, commit and copy at its far end."""
    torch = torch_mod()
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    hd, H, Hkv, n = 128, 4, 2, 20
    pages = (1 << 32) // (Hkv * 16 * hd) + 64  # 8.6 GB a pool
    pool = torch.zeros((2, pages, Hkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    table = np.array([[pages - 1, 3, pages - 17]], np.int32)
    view = fp.fp_kv_view(0, Hkv, hd, 16, 3, pages, pool[0].data_ptr(), pool[1].data_ptr(), None, None, ptr(dev(table)))
    qkv = synth.uniform_bf16(5, 1, (n, (H + 2 * Hkv) * hd), -2, 2)
    cu, pos, err = dev(np.array([0, n], np.int32)), dev(np.array([13], np.int32)), empty(1, np.int32)
    path = [0, 2, 3, 9, 15, 19]
    fp.fp_op_rope_kv_tree(ptr(dev(qkv)), qkv.shape[1], n, 1, H, view, ptr(cu), ptr(pos), ptr(dev(np.zeros(n, np.int32))),
                          ptr(_table(fp, 3, hd)), ptr(empty((n, H * hd), np.uint16)), H * hd, ptr(err))
    fp.fp_op_kv_commit(view, n, 1, ptr(cu), ptr(pos), ptr(dev(np.array(path + [-1] * 14, np.int32))), ptr(err))
    fp.fp_op_kv_copy(view, 1, ptr(dev(np.array([pages - 1], np.int32))), ptr(dev(np.array([pages - 5], np.int32))),
                     ptr(dev(np.array([16], np.int32))), ptr(err))
    assert host(err, np.int32)[0] == 0
    v = qkv.reshape(n, -1, hd)[:, H + Hkv :]
    for j, r in enumerate(path):
        page, slot = int(table[0, (13 + j) // 16]), (13 + j) % 16
        assert np.array_equal(pool[1, page, :, slot].view(torch.int16).cpu().numpy().view(np.uint16), v[r]), j
        if page == pages - 1:
            assert torch.equal(pool[:, pages - 5, :, slot], pool[:, page, :, slot])


# ------------------------------------------------------------------ a whole step
@pytest.mark.parametrize("kvq", [0, 1])
@pytest.mark.parametrize("graph", [False, True])
def test_a_step_as_it_is_used(fp, kvq, graph):
    """Plan, append, attend, probabilities, verify, commit, on one stream, eager and as one captured graph: every row
    attends to its own branch, and afterwards the cache holds the accepted tokens as if they had been appended in a row."""
    torch = torch_mod()
    H, Hkv, hd, V = 8, 2, 128, 500
    seqs = [(16, 100), (1, 7), (40, 250)]
    c = Trees(fp, kvq, hd, H, Hkv, seqs, 43)
    rng = np.random.default_rng(8)
    qkv = synth.uniform_bf16(6, 1, (c.N, (H + 2 * Hkv) * hd), -1.5, 1.5)
    logits = rng.normal(size=(c.N, V)).astype(np.float32)
    tokens = c.flat([[0] * n for n, _ in seqs], 0)
    for b, t in enumerate(c.parents):  # the first two children of a row carry its likeliest tokens
        born = {}
        for i, p in enumerate(t[1:], 1):
            at = born.setdefault(p, [])
            tokens[c.cu[b] + i] = (37 * p + 5 * len(at)) % V
            logits[c.cu[b] + p, tokens[c.cu[b] + i]] = 8.0 - len(at)
            at.append(i)
    u = rng.random(c.N).astype(np.float32)
    st = torch.cuda.Stream()
    words = c.words
    d = {"qkv": dev(qkv), "logits": dev(logits), "tokens": dev(tokens), "u": dev(u), "cu": dev(c.cu), "pos": dev(c.pos),
         "parent": dev(c.flat(c.parents)), "depth": empty(c.N, np.int32), "mask": empty((c.N, words), np.int32),
         "q": empty((c.N, H * hd), np.uint16), "o": empty((c.N, H * hd), np.uint16), "p": empty((c.N, V), np.float32),
         "path": empty(c.N, np.int32), "out": empty(c.N, np.int32), "cnt": empty(c.B, np.int32), "err": empty(1, np.int32),
         "cs": _table(fp, c.pps, hd)}
    need = fp.fp_op_attention_tree_workspace_bytes(c.B, H, Hkv, hd, c.max_new)
    ws = empty(need + 256)
    P = {k: ptr(x) for k, x in d.items()}

    def step():
        s = st.cuda_stream
        fp.fp_op_tree_plan(P["parent"], c.N, c.B, P["cu"], c.max_new, P["depth"], P["mask"], words, P["err"], s)
        fp.fp_op_rope_kv_tree(P["qkv"], qkv.shape[1], c.N, c.B, H, c.view, P["cu"], P["pos"], P["depth"], P["cs"], P["q"],
                              H * hd, P["err"], s)
        fp.fp_op_attention_tree(P["q"], H * hd, c.N, c.B, H, c.view, P["cu"], P["pos"], P["mask"], words, c.max_new, c.max_len,
                                P["o"], (ptr(ws) + 255) // 256 * 256, need, P["err"], s)
        fp.fp_op_softmax(P["logits"], c.N, V, None, P["p"], P["err"], s)
        fp.fp_op_verify_tree(P["p"], V, c.N, c.B, P["cu"], P["parent"], P["tokens"], P["u"], P["path"], P["out"], P["cnt"],
                             P["err"], s)
        fp.fp_op_kv_commit(c.view, c.N, c.B, P["cu"], P["pos"], P["path"], P["err"], s)

    torch.cuda.synchronize()
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            step()
        for _ in range(2):  # (a step begins by writing every row that it reads)
            g.replay()
    else:
        step()
    torch.cuda.synchronize()
    assert host(d["err"], np.int32)[0] == 0
    # the verification, against the probabilities that the GPU made
    p = host(d["p"], np.float32).reshape(c.N, V)
    want = _expected(p, c.cu, c.flat(c.parents), tokens, u)
    path, out, cnt = host(d["path"], np.int32), host(d["out"], np.int32), host(d["cnt"], np.int32)
    _same((path, out, cnt), want[:3])
    assert cnt.max() > 2
    # the cache before the commit, from a second append into a copy; then the attention over it
    c2 = Trees(fp, kvq, hd, H, Hkv, seqs, 43)
    depth = c.flat([several.plan(t)[0] for t in c.parents])
    _, err = _append(c2, qkv, depth)
    assert err == 0
    c2.data = {w: host(t, c2.data[w].dtype).reshape(c2.data[w].shape).copy() for w, t in c2.dev.items()}
    c2.check(host(d["q"], np.uint16).reshape(c.N, -1), host(d["o"], np.uint16).reshape(c.N, -1))
    after = _committed(c2, [path[c.cu[b] : c.cu[b] + cnt[b]].tolist() for b in range(c.B)])
    for w in after:
        assert np.array_equal(host(c.dev[w], after[w].dtype).reshape(after[w].shape).view(np.uint8), after[w].view(np.uint8)), w
    # the accepted rows appended one after another, as a chunk, into a fresh cache: the same bits
    for b in range(c.B):
        rows = c.cu[b] + path[c.cu[b] : c.cu[b] + cnt[b]]
        line = Batch(fp, kvq, hd, H, Hkv, [(len(rows), seqs[b][1])], 1)
        q, err2 = empty((len(rows), H * hd), np.uint16), empty(1, np.int32)
        fp.fp_op_rope_kv_chunk(ptr(dev(qkv[rows])), qkv.shape[1], len(rows), 1, H, line.view, ptr(dev(line.cu)),
                               ptr(dev(line.pos)), ptr(_table(fp, line.pps, hd)), ptr(q), H * hd, ptr(err2))
        assert host(err2, np.int32)[0] == 0
        now = {w: host(t, line.data[w].dtype).reshape(line.data[w].shape) for w, t in line.dev.items()}
        for j in range(len(rows)):
            t = seqs[b][1] + j
            for w in now:
                assert np.array_equal(now[w][line.table[0, t // 16], :, t % 16], after[w][c.table[b, t // 16], :, t % 16]), (w, b, j)
