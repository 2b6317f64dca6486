"""Beams against the oracle: selection, reordering of page tables, copies of pages, and a whole search.

A candidate's value is score + x - lse.  The sum is held in pairs of fp32 and rounded once, 2^-24 |value|; the normaliser
errs by its exponentials (ex2.approx: 2^-22 each) and the roundings of its sum (at most 25 additions one after another
for rows of up to 16384 values a piece, 2^-24 each) and logarithm (2^-24): 2^-22 + 27 * 2^-24 < 2^-19.  So
    |score - value| <= 2^-24 |value| + 2^-19,
and two candidates of different beams whose values differ by more than 2^-18 come in their order; of one beam, always.
"""
import numpy as np
import pytest

import synth
from oracle import quant, several
from tests.gpu_helpers import dev, empty, host, ptr, torch_mod
from tests.test_gpu_chunk import Batch

pytestmark = pytest.mark.gpu

LSE = 2.0 ** -19


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _select(fp, x, B, W, score, done=None, end=-1, ws=None, in_place=False, offset=0, stream=None):
    V = x.shape[1]
    xd = empty(x.size + offset, np.float32)
    xd[offset:] = dev(x).reshape(-1)
    need = fp.fp_op_beam_select_workspace_bytes(B, W, V)
    if ws is None:
        ws = empty(need + 256)
        ws[65536 + 256:] = 255
    sd, dd = dev(score.astype(np.float32)), None if done is None else dev(np.array(done, np.int32))
    out = sd if in_place else dev(np.full(B * W, 55, np.float32))
    nd = dd if in_place else dev(np.full(B * W, 55, np.int32))
    par, tok, err = dev(np.full(B * W, 55, np.int32)), dev(np.full(B * W, 55, np.int32)), empty(1, np.int32)
    fp.fp_op_beam_select(ptr(xd) + 4 * offset, V, B, W, ptr(sd), ptr(dd), end, ptr(par), ptr(tok), ptr(out), ptr(nd),
                         (ptr(ws) + 255) // 256 * 256, need, ptr(err), stream)
    return (host(par, np.int32), host(tok, np.int32), host(out, np.float32),
            None if nd is None else host(nd, np.int32), int(host(err, np.int32)[0]))


def _check(got, x, B, W, score, done=None, end=-1):
    par, tok, new, nd, err = got
    done = np.zeros(B * W, int) if done is None else np.array(done)
    good = True
    for b in range(B):
        r = slice(b * W, b * W + W)
        want, ok = several.select(x[r], score[r], done[r], end)
        good &= ok
        lse = {}
        for w in range(W):
            z = x[b * W + w].astype(np.float64)
            m = z.max()
            with np.errstate(all="ignore"):
                lse[w] = m + np.log(np.exp(z - m).sum())
        for c, (pw, pt, ps, pd) in enumerate(want):
            o = b * W + c
            gw, gt = int(par[o]), int(tok[o])
            if pw < 0:
                assert (gw, gt) == (-1, -1) and new[o] == -np.inf and (nd is None or nd[o] == 0), (b, c)
                continue
            # what was chosen has the value it should have in this place
            v = float(score[b * W + gw]) + (0.0 if done[b * W + gw] else float(x[b * W + gw, gt]) - lse[gw])
            assert abs(v - ps) <= 2 * LSE, (b, c, gw, gt, want[c])
            if abs(v - ps) > 0 or gw == pw:
                assert gw != pw or gt == pt, (b, c)
            near = [abs(ps - q[2]) <= 2 * LSE and q[0] != pw for q in want]
            if not any(near) and c < W - 1:
                assert (gw, gt) == (pw, pt), (b, c, (gw, gt), want[c])
            assert abs(new[o] - v) <= 2.0 ** -24 * abs(v) + LSE, (b, c, new[o], v)
            if nd is not None:
                assert nd[o] == int(bool(done[b * W + gw]) or gt == end)
        assert len({(int(par[o]), int(tok[o])) for o in range(b * W, b * W + W) if par[o] >= 0}) == sum(w[0] >= 0 for w in want)
    assert err == int(not good)


SHAPES = [(1, 1, 1), (1, 1, 2), (3, 2, 3), (2, 4, 33), (1, 8, 1000), (5, 3, 4097), (2, 5, 16385), (32, 4, 32000),
          (1, 8, 128001), (2, 32, 5000), (1, 32, 70001), (7, 16, 517), (1, 1, 300000), (1, 2, 600011), (40, 10, 999), (2, 8, 3),
          (3, 32, 1), (600, 2, 90)]


@pytest.mark.parametrize("B,W,V", SHAPES)
def test_select(fp, B, W, V):
    rng = np.random.default_rng(B * 1000 + W + V)
    x = (3 * rng.normal(size=(B * W, V))).astype(np.float32)
    x[:, 7::97] = -np.inf
    score = (-6 * rng.random(B * W)).astype(np.float32)
    _check(_select(fp, x, B, W, score), x, B, W, score)
    done = rng.random(B * W) < 0.3
    end = min(2, V - 1)
    _check(_select(fp, x, B, W, score, done, end, in_place=True, offset=1), x, B, W, score, done, end)


@pytest.mark.parametrize("B,W,V", [(2, 4, 1000), (1, 8, 40001), (1, 32, 700), (1, 1, 33000)])
@pytest.mark.parametrize("how", ["constant", "steps", "rising", "falling"])
def test_select_ties_and_orders(fp, how, B, W, V):
    """Equal logits, few distinct ones, sorted ones: ties to the lowest beam, then token, exactly."""
    rng = np.random.default_rng(V)
    x = {"constant": np.zeros((B * W, V)), "steps": rng.integers(0, 4, (B * W, V)) * 0.5,
         "rising": np.tile(np.arange(V) / 64.0, (B * W, 1)), "falling": np.tile(-np.arange(V) / 64.0, (B * W, 1))}[how]
    x = x.astype(np.float32)
    x[:] = x[:1]  # the same row for every beam, so equal scores tie across beams
    score = np.repeat(-rng.random(B), W).astype(np.float32)
    got = _select(fp, x, B, W, score)
    order = np.lexsort((np.arange(V), -x[0]))[:W]
    v = x[0, order]
    every = sorted((-float(v[i]), w, int(order[i])) for w in range(W) for i in range(len(order)))[:W]
    for b in range(B):
        assert [(int(got[0][b * W + c]), int(got[1][b * W + c])) for c in range(W)] == [(w, t) for _, w, t in every], b
    assert got[4] == 0


def test_select_same_value_in_negative_zero(fp):
    x = np.full((1, 100), -5.0, np.float32)
    x[0, [90, 40]] = 0.0
    x[0, [60, 10]] = -0.0
    got = _select(fp, np.repeat(x, 4, 0), 1, 4, np.array([-1.0, -np.inf, -np.inf, -np.inf], np.float32))
    assert got[1].tolist() == [10, 40, 60, 90] and got[0].tolist() == [0] * 4


def test_select_from_one_prompt(fp):
    """The first step: only beam 0 exists, all continuations are its own."""
    rng = np.random.default_rng(0)
    for W in (2, 7, 32):
        x = rng.normal(size=(3 * W, 2000)).astype(np.float32)
        score = np.where(np.arange(3 * W) % W == 0, 0.0, -np.inf).astype(np.float32)
        got = _select(fp, x, 3, W, score)
        _check(got, x, 3, W, score)
        assert np.all(got[0] == 0)


def test_select_without_enough_candidates(fp):
    """Ended, dead and banned: places without a candidate."""
    W, V = 4, 50
    x = np.full((3 * W, V), -np.inf, np.float32)
    x[0, 3] = 1.0
    x[5, :2] = 0.0
    score = np.array([-1, -np.inf, -np.inf, -2, -1, -3, -np.inf, -np.inf] + [-np.inf] * 4, np.float32)
    done = [0, 1, 0, 1] + [0] * 8
    got = _select(fp, x, 3, W, score, done, 9)
    _check(got, x, 3, W, score, done, 9)
    assert got[4] == 0 and got[0][:4].tolist() == [0, 3, -1, -1] and got[1][:4].tolist() == [3, 9, -1, -1]


@pytest.mark.parametrize("what", [np.nan, np.inf])
def test_select_reports_what_is_not_finite(fp, what):
    """A NaN or +inf leaves its beam without candidates; in an ended or dead beam it is not read; scores likewise."""
    rng = np.random.default_rng(1)
    W, V = 4, 40000
    x = rng.normal(size=(2 * W, V)).astype(np.float32)
    score = (-rng.random(2 * W)).astype(np.float32)
    x[1, 39999] = what
    _check(_select(fp, x, 2, W, score), x, 2, W, score)
    done = np.arange(2 * W) == 1
    got = _select(fp, x, 2, W, score, done, 3)
    _check(got, x, 2, W, score, done, 3)
    assert got[4] == 0
    score[1] = -np.inf
    assert _select(fp, x, 2, W, score)[4] == 0
    score[6] = what
    got = _select(fp, x, 2, W, score)
    _check(got, x, 2, W, score)
    assert got[4] == 1


def test_select_large_and_far_logits(fp):
    """Logits of thousands, a far row beside a near one, a spread over hundreds: the normaliser holds."""
    rng = np.random.default_rng(2)
    W, V = 4, 9000
    x = rng.normal(size=(W, V)).astype(np.float32)
    x[0] += 5000
    x[1] -= 70000
    x[2] *= 200
    score = np.array([-1.0, -1.5, -2.0, -0.5], np.float32)
    got = _select(fp, x, 1, W, score)
    # logits near 5000 are multiples of 2^-11: their differences are exact, the pairs carry the rest
    _check(got, x, 1, W, score)


def test_select_repeats_and_leaves_its_tickets_clear(fp):
    """One workspace for calls of several shapes in turn, eager and captured; the same bits each time."""
    torch = torch_mod()
    shapes = [(4, 8, 20000), (1, 4, 1000), (9, 2, 64000), (2, 32, 3001)]
    need = max(fp.fp_op_beam_select_workspace_bytes(*s) for s in shapes)
    ws = empty(need + 256)
    first = {}
    for turn in range(3):
        for B, W, V in shapes:
            rng = np.random.default_rng(V)
            x, score = rng.normal(size=(B * W, V)).astype(np.float32), (-rng.random(B * W)).astype(np.float32)
            got = _select(fp, x, B, W, score, ws=ws)
            if turn == 0:
                _check(got, x, B, W, score)
                first[V] = got
            for a, z in zip(got, first[V]):
                assert np.array_equal(a, z)
    at = -ptr(ws) % 256
    assert not host(ws, np.uint8)[at:at + 65536].any()
    # a captured call, replayed on other logits
    B, W, V = 4, 8, 20000
    x, score = empty((B * W, V), np.float32), empty(B * W, np.float32)
    out = [empty(B * W, np.int32), empty(B * W, np.int32), empty(B * W, np.float32), empty(B * W, np.int32), empty(1, np.int32)]
    st = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=st):
        fp.fp_op_beam_select(ptr(x), V, B, W, ptr(score), None, -1, *[ptr(o) for o in out[:4]], (ptr(ws) + 255) // 256 * 256,
                             need, ptr(out[4]), st.cuda_stream)
    for seed in range(3):
        rng = np.random.default_rng(seed)
        xs, sc = rng.normal(size=(B * W, V)).astype(np.float32), (-rng.random(B * W)).astype(np.float32)
        x.copy_(torch.from_numpy(xs))
        score.copy_(torch.from_numpy(sc))
        g.replay()
        torch.cuda.synchronize()
        _check((host(out[0], np.int32), host(out[1], np.int32), host(out[2], np.float32), host(out[3], np.int32),
                int(host(out[4], np.int32)[0])), xs, B, W, sc)


# ------------------------------------------------------------------ reordering and copies
def _reorder(fp, tables, lens, parents):
    B, W, pps = tables.shape
    out = [dev(np.full((B * W, pps), 55, np.int32))] + [dev(np.full(B * W, 55, np.int32)) for _ in range(3)]
    err = empty(1, np.int32)
    fp.fp_op_beam_reorder(B, W, pps, 16, ptr(dev(np.array(lens, np.int32))), ptr(dev(np.array(parents, np.int32))),
                          ptr(dev(tables.astype(np.int32))), *[ptr(o) for o in out], ptr(err))
    h = [host(o, np.int32) for o in out]
    return h[0].reshape(B, W, pps), np.stack(h[1:], -1).reshape(B, W, 3), int(host(err, np.int32)[0])


@pytest.mark.parametrize("B,W,pps", [(1, 1, 1), (3, 4, 5), (20, 32, 9), (5, 7, 300), (2, 31, 2)])
def test_reorder(fp, B, W, pps):
    rng = np.random.default_rng(W)
    for turn in range(4):
        tables = rng.permutation(B * W * pps).reshape(B, W, pps)
        lens = rng.integers(0, pps * 16 + 1, B)
        if turn == 1:
            lens = lens // 16 * 16
        if turn == 2:
            lens[:] = pps * 16
        parents = rng.integers(-1 if turn == 3 else 0, W, (B, W))
        if turn == 2:
            parents[:] = W - 1
        new, copies, err = _reorder(fp, tables, lens, parents)
        assert err == 0
        for b in range(B):
            n, c, _ = several.reorder(tables[b], int(lens[b]), parents[b].tolist())
            assert np.array_equal(new[b], n) and copies[b].tolist() == [list(x) for x in c], (turn, b)


def test_reorder_reports_bad_lengths_and_parents(fp):
    tables = np.arange(3 * 4 * 2).reshape(3, 4, 2)
    parents = np.array([[3, 3, 3, 3], [1, 4, -2, 2 ** 31 - 1], [0, 0, 1, 1]])
    for lens in ([33, 17, 9], [-1, 17, 9]):
        new, copies, err = _reorder(fp, tables, lens, parents)
        assert err == 1
        for b in range(3):
            n, c, _ = several.reorder(tables[b], lens[b], parents[b].tolist())
            assert np.array_equal(new[b], n) and copies[b].tolist() == [list(x) for x in c], b


@pytest.mark.parametrize("kvq,hd,Hkv", [(0, 128, 8), (1, 128, 8), (0, 64, 5), (1, 64, 3), (0, 128, 40), (1, 64, 1)])
def test_copy(fp, kvq, hd, Hkv):
    """Rows 0 to 16 of pages: all bits of the pools."""
    c = Batch(fp, kvq, hd, Hkv, Hkv, [(1, 900)], 3)
    rng = np.random.default_rng(Hkv)
    pages = rng.permutation(c.pages)[:50].astype(np.int32)
    src, dst = pages[:25].copy(), pages[25:].copy()
    src[4] = src[5]  # one page to two
    rows = np.arange(25).astype(np.int32) % 17
    src[7] = -1
    err = empty(1, np.int32)
    fp.fp_op_kv_copy(c.view, 25, ptr(dev(src)), ptr(dev(dst)), ptr(dev(rows)), ptr(err))
    assert host(err, np.int32)[0] == 0
    want = {w: x.copy() for w, x in c.data.items()}
    for a, z, n in zip(src, dst, rows):
        if a >= 0:
            for w in want:
                want[w][z, :, :n] = c.data[w][a, :, :n]
    for w in want:
        assert np.array_equal(host(c.dev[w], want[w].dtype).reshape(want[w].shape).view(np.uint8), want[w].view(np.uint8)), w


def test_copy_reports_and_skips_bad_pages(fp):
    c = Batch(fp, 1, 64, 2, 2, [(1, 100)], 5)
    src, dst, rows = [-2, c.pages, 0, 1, 2, 3], [1, 1, c.pages, -1, 4, 5], [3, 3, 3, 3, 17, -1]
    for i in range(6):
        err = empty(1, np.int32)
        fp.fp_op_kv_copy(c.view, 1, ptr(dev(np.array(src[i:i + 1], np.int32))), ptr(dev(np.array(dst[i:i + 1], np.int32))),
                         ptr(dev(np.array(rows[i:i + 1], np.int32))), ptr(err))
        assert host(err, np.int32)[0] == 1, i
    for w in c.data:
        assert np.array_equal(host(c.dev[w], c.data[w].dtype).reshape(c.data[w].shape), c.data[w])


def test_a_captured_step_of_beams(fp):
    """Select, reorder, copy, twice, as one graph on one stream: replayed on other logits and lengths, the tables and the
    pools are the oracle's of what the selection chose."""
    torch = torch_mod()
    B, W, V, pps, hd, Hkv = 3, 5, 3001, 7, 64, 2
    R, pages = B * W, B * W * pps
    c = Batch(fp, 1, hd, Hkv, Hkv, [(1, pages * 16 - 1)], 11)
    pools = {w: c.dev[w].clone() for w in c.data}
    x, score, lens = [empty((R, V), np.float32) for _ in range(2)], [empty(R, np.float32) for _ in range(3)], empty(B, np.int32)
    par, tok = [empty(R, np.int32) for _ in range(2)], empty(R, np.int32)
    tabs, lists, err = [empty((R, pps), np.int32) for _ in range(3)], [[empty(R, np.int32) for _ in range(3)] for _ in range(2)], empty(1, np.int32)
    need = fp.fp_op_beam_select_workspace_bytes(B, W, V)
    ws = empty(need + 256)
    st = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=st):
        s = st.cuda_stream
        for i in range(2):
            fp.fp_op_beam_select(ptr(x[i]), V, B, W, ptr(score[i]), None, -1, ptr(par[i]), ptr(tok), ptr(score[i + 1]), None,
                                 (ptr(ws) + 255) // 256 * 256, need, ptr(err), s)
            fp.fp_op_beam_reorder(B, W, pps, 16, ptr(lens), ptr(par[i]), ptr(tabs[i]), ptr(tabs[i + 1]),
                                  *[ptr(o) for o in lists[i]], ptr(err), s)
            fp.fp_op_kv_copy(c.view, R, *[ptr(o) for o in lists[i]], ptr(err), s)
    for seed in range(4):
        rng = np.random.default_rng(seed)
        xs = rng.normal(size=(2, R, V)).astype(np.float32)
        length = rng.integers(0, pps * 16, B).astype(np.int32)
        table = rng.permutation(pages).reshape(R, pps).astype(np.int32)
        first = (-5 * rng.random(R)).astype(np.float32)
        for w in pools:
            c.dev[w].copy_(pools[w])
        for a, z in ((x[0], xs[0]), (x[1], xs[1]), (lens, length), (tabs[0], table), (score[0], first)):
            a.copy_(torch.from_numpy(z))
        g.replay()
        torch.cuda.synchronize()
        assert host(err, np.int32)[0] == 0
        want = {w: v.copy() for w, v in c.data.items()}
        for i in range(2):
            chosen = host(par[i], np.int32).reshape(B, W)
            sums = host(score[i], np.float32).astype(np.float64)
            z = xs[i].astype(np.float64)
            best = np.sort((sums[:, None] + z - np.log(np.exp(z).sum(1))[:, None]).reshape(B, W * V), 1)[:, ::-1][:, :W]
            new = host(score[i + 1], np.float32).reshape(B, W)
            assert np.all(np.abs(new - best) <= 2.0 ** -24 * np.abs(best) + LSE)
            for b in range(B):
                t, copies, _ = several.reorder(table.reshape(B, W, pps)[b], int(length[b]), chosen[b].tolist())
                table.reshape(B, W, pps)[b] = t
                assert [list(v) for v in copies] == np.stack([host(o, np.int32) for o in lists[i]], -1)[b * W:b * W + W].tolist()
                for a, z1, n in copies:
                    for w in want:
                        if n:
                            want[w][z1, :, :n] = want[w][a, :, :n]
            assert np.array_equal(host(tabs[i + 1], np.int32).reshape(R, pps), table)
        for w in want:
            assert np.array_equal(host(c.dev[w], want[w].dtype).reshape(want[w].shape).view(np.uint8), want[w].view(np.uint8)), w


@pytest.mark.parametrize("kvq", [0, 1])
def test_a_search_as_it_is_used(fp, kvq):
    """Forty steps of two layers: append the beams' tokens, attend over each beam's own history, select, reorder, copy.
    Selection against the oracle at every step; the caches hold each hypothesis' own rows, and attention over them is
    the oracle's, at the end."""
    torch = torch_mod()
    B, W, H, Hkv, hd, V, L = 2, 4, 4, 2, 64, 1000, 2
    start, steps = [21, 30], 40
    pps = 6
    rng = np.random.default_rng(kvq)
    pages = B * W * pps
    table = rng.permutation(pages).reshape(B * W, pps).astype(np.int32)
    dt = np.uint16 if kvq == 0 else np.int8
    pools = [{w: empty((pages, Hkv, 16, hd), dt) for w in "kv"} | {w + "s": empty((pages, Hkv, 16), np.float32) for w in "kv"} for _ in range(L)]
    tabs = [dev(table), empty((B * W, pps), np.int32)]
    cs = empty((pps * 16, hd // 2, 2), np.float32)
    fp.fp_op_rope_table(pps * 16, hd, 10000.0, ptr(cs))
    err, ws_b = empty(1, np.int32), fp.fp_op_beam_select_workspace_bytes(B, W, V)
    ws = empty(ws_b + 256)
    need = fp.fp_op_attention_chunk_workspace_bytes(B * W, H, Hkv, hd, 64)
    aws = empty(need + 256)
    aws_p, ws_p = ((ptr(x) + 255) // 256 * 256 for x in (aws, ws))
    row = (H + 2 * Hkv) * hd

    def view(layer, which):
        p = pools[layer]
        return fp.fp_kv_view(kvq, Hkv, hd, 16, pps, pages, ptr(p["k"]), ptr(p["v"]), ptr(p["ks"]), ptr(p["vs"]), ptr(tabs[which]))

    def qkv_of(layer, b, text):  # a token's rows, by its place and what came before it
        return synth.uniform_bf16(31 * layer + b, 7 + hash(text) % 100003, (1, row), -1.5, 1.5)[0]

    # prompts, in beam 0's pages
    texts = [[tuple((b, i) for i in range(start[b]))] * W for b in range(B)]
    texts = [[t[0]] + [()] * (W - 1) for t in texts]
    for layer in range(L):
        rows = np.stack([qkv_of(layer, b, texts[b][0][: i + 1]) for b in range(B) for i in range(start[b])])
        cu = np.zeros(B * W + 1, np.int32)
        cu[1:] = np.cumsum([start[b] if w == 0 else 0 for b in range(B) for w in range(W)])
        q = empty((len(rows), H * hd), np.uint16)
        fp.fp_op_rope_kv_chunk(ptr(dev(rows)), row, len(rows), B * W, H, view(layer, 0), ptr(dev(cu)),
                               ptr(dev(np.zeros(B * W, np.int32))), ptr(cs), ptr(q), H * hd, ptr(err))
    score = np.where(np.arange(B * W) % W == 0, 0.0, -np.inf).astype(np.float32)
    sd = dev(score)
    dd = dev(np.zeros(B * W, np.int32))
    par, tok = empty(B * W, np.int32), empty(B * W, np.int32)
    copies = [empty(B * W, np.int32) for _ in range(3)]
    which, last = 0, None
    cu1 = dev(np.arange(B * W + 1, dtype=np.int32))
    for step in range(steps):
        n = [s + step for s in start]
        x = (2.5 * rng.normal(size=(B * W, V))).astype(np.float32)
        before, ended = host(sd, np.float32).copy(), host(dd, np.int32).copy()
        fp.fp_op_beam_select(ptr(dev(x)), V, B, W, ptr(sd), ptr(dd), 5, ptr(par), ptr(tok), ptr(sd), ptr(dd), ws_p, ws_b, ptr(err))
        p, t = host(par, np.int32), host(tok, np.int32)
        _check((p, t, host(sd, np.float32), host(dd, np.int32), int(host(err, np.int32)[0])), x, B, W, before, ended, 5)
        lens = np.array(n, np.int32)
        fp.fp_op_beam_reorder(B, W, pps, 16, ptr(dev(lens)), ptr(par), ptr(tabs[which]), ptr(tabs[1 - which]),
                              *[ptr(c) for c in copies], ptr(err))
        which = 1 - which
        texts = [[texts[b][p[b * W + w]] + ((int(t[b * W + w]), step),) for w in range(W)] for b in range(B)]
        for layer in range(L):
            v = view(layer, which)
            fp.fp_op_kv_copy(v, B * W, *[ptr(c) for c in copies], ptr(err))
            rows = np.stack([qkv_of(layer, b, texts[b][w]) for b in range(B) for w in range(W)])
            q, o = empty((B * W, H * hd), np.uint16), empty((B * W, H * hd), np.uint16)
            pos = dev(np.repeat(lens, W))
            fp.fp_op_rope_kv_chunk(ptr(dev(rows)), row, B * W, B * W, H, v, ptr(cu1), ptr(pos), ptr(cs), ptr(q), H * hd, ptr(err))
            fp.fp_op_attention_chunk(ptr(q), H * hd, B * W, B * W, H, v, ptr(cu1), ptr(pos), 1, pps * 16, ptr(o), aws_p, need,
                                     ptr(err))
            last = (q, o)
    assert host(err, np.int32)[0] == 0
    torch.cuda.synchronize()
    # each hypothesis' rows, rebuilt in a cache of its own
    tb = host(tabs[which], np.int32).reshape(B * W, pps)
    for b in range(B):
        for w in range(W):
            text, r = texts[b][w], b * W + w
            for layer in range(L):
                rows = np.stack([qkv_of(layer, b, text[: i + 1]) for i in range(len(text))])
                line = Batch(fp, kvq, hd, H, Hkv, [(len(rows), 0)], 1)
                q = empty((len(rows), H * hd), np.uint16)
                fp.fp_op_rope_kv_chunk(ptr(dev(rows)), row, len(rows), 1, H, line.view, ptr(dev(line.cu)), ptr(dev(line.pos)),
                                       ptr(cs), ptr(q), H * hd, ptr(err))
                line.data = {k: host(x, line.data[k].dtype).reshape(line.data[k].shape) for k, x in line.dev.items()}
                i = np.arange(len(rows))
                for k in line.data:
                    mine = host(pools[layer][k], line.data[k].dtype).reshape((pages,) + line.data[k].shape[1:])
                    assert np.array_equal(mine[tb[r, i // 16], :, i % 16], line.data[k][line.table[0, i // 16], :, i % 16]), (b, w, layer, k)
                if layer == L - 1:
                    k, v = line.cached("k", 0, len(rows)), line.cached("v", 0, len(rows))
                    xq = quant.bf16_to_f32(host(last[0], np.uint16).reshape(B * W, H, hd)[r : r + 1]).astype(np.float64)
                    got = quant.bf16_to_f32(host(last[1], np.uint16).reshape(B * W, H, hd)[r : r + 1])
                    vis = np.ones((1, len(rows)), bool)
                    ref, mass = several.attention(xq, vis, k, v), several.attention(xq, vis, k, np.abs(v))
                    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * mass + 1e-30)
