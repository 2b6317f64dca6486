"""Probabilities and the verification of drafted tokens against the oracle, and a drafted step as a whole."""
import numpy as np
import pytest

import synth
from oracle import chunk
from oracle import model as M
from oracle import quant
from tests.gpu_helpers import dev, empty, host, ptr, torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


def _softmax(fp, x, temp=None, in_place=False, shift=0):
    """fp_op_softmax of x [M][V], its buffers `shift` floats off a 16-byte boundary."""
    M_, V = x.shape
    buf = dev(np.concatenate([np.zeros(shift, np.float32), x.reshape(-1), np.full(4, 7.0, np.float32)]))
    out = buf if in_place else dev(np.full(M_ * V + shift + 4, 7.0, np.float32))
    err = empty(1, np.int32)
    fp.fp_op_softmax(ptr(buf) + 4 * shift, M_, V, ptr(dev(np.asarray(temp, np.float32))) if temp is not None else None,
                     ptr(out) + 4 * shift, ptr(err))
    y = host(out, np.float32)
    assert np.all(y[shift + M_ * V:] == 7.0)
    return y[shift:shift + M_ * V].reshape(M_, V), int(host(err, np.int32)[0])


def _check_probs(got, x, temp=None):
    """y = e^z / sum e^z, z = (x - max) / T.  In fp32 z carries three roundings (3 2^-24 |z|), 2^z two units (2^-22),
    the sum one rounding a term of a thread's run and a few more (run up to 64: 2^-17); below 2^-126 zero."""
    ref = chunk.probabilities(x, temp)
    t = np.ones(len(x)) if temp is None else np.asarray(temp, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        z = np.where(np.isfinite(x), np.abs(x.astype(np.float64) - x.max(-1, keepdims=True)), 0) / np.where(t > 0, t, 1)[:, None]
    assert np.all(np.abs(got - ref) <= ref * (2.0 ** -17 + 3 * 2.0 ** -24 * z) + 2.0 ** -126)


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("m,V", [(1, 1), (3, 2), (5, 31), (4, 1000), (7, 4099), (160, 32000), (3, 128001), (1, 300007),
                                 (2, 1100003)])
def test_softmax(fp, m, V, shift):
    if shift and V > 200000:
        pytest.skip("one alignment of the longest rows is enough")
    rng = np.random.default_rng(V + m)
    x = (4 * rng.standard_normal((m, V))).astype(np.float32)
    x[:, 1::7] = -np.inf if V > 10 else x[:, 1::7]
    temp = rng.uniform(0.3, 2.0, m).astype(np.float32)
    for t in (None, temp):
        got, err = _softmax(fp, x, t, shift=shift)
        assert err == 0
        _check_probs(got, x, t)
    got, _ = _softmax(fp, x, temp, in_place=True, shift=shift)
    _check_probs(got, x, temp)


def test_softmax_special_rows(fp):
    V = 777
    rng = np.random.default_rng(2)
    x = rng.standard_normal((10, V)).astype(np.float32)
    x[0] = -np.inf                              # nothing left
    x[1, :] = -np.inf
    x[1, 700] = -3e38                           # one token left
    x[2, [5, 400, 776]] = 50.0                  # greedy tie: the lowest
    x[3] = 88.0                                 # uniform
    x[4, 3] = np.nan
    x[5, 3] = np.inf
    x[6] = np.linspace(-3.4e38, 3.4e38, V)      # the whole range of fp32
    x[9] = -np.inf
    t = np.array([1, 1, 0, 1, 1, 1, 1, 1e-30, 1, 0], np.float32)
    got, err = _softmax(fp, x, t)
    assert err == 0
    assert np.all(got[0] == 0) and np.all(got[9] == 0)
    assert got[1].sum() == got[1, 700] == 1
    assert got[2].sum() == got[2, 5] == 1
    assert np.all(np.abs(got[3] * V - 1) <= 2.0 ** -17)
    assert np.all(np.isnan(got[4])) and np.all(np.isnan(got[5]))
    assert got[6].sum() == got[6, V - 1] == 1
    assert got[7].sum() == got[7, x[7].argmax()] == 1
    _check_probs(got[8:9], x[8:9])
    y = np.full((2, V), -np.inf, np.float32)  # a NaN among masked tokens; with T = 0 it is not the largest
    y[:, 500] = np.nan
    y[1, 600] = 1.0
    got, err = _softmax(fp, y, np.array([1, 0], np.float32))
    assert err == 0 and np.all(np.isnan(got[0])) and got[1].sum() == got[1, 600] == 1
    for bad in (-1.0, np.nan, np.inf, -np.inf):
        got, err = _softmax(fp, x[6:9], np.array([1, bad, 1], np.float32))
        assert err == 1 and np.all(got[1] == 0)
        _check_probs(got[2:], x[8:9])


# ------------------------------------------------------------------ verification
def _verify(fp, p, q, tokens, u, r, cu, B, stream=None):
    N, V = p.shape
    out, cnt = dev(np.full(N + 2, -7, np.int32)), dev(np.full(B, -7, np.int32))
    err = empty(1, np.int32)
    fp.fp_op_verify_draft(ptr(dev(p)), ptr(dev(q)) if q is not None else None, V, N, B, ptr(dev(np.asarray(cu, np.int32))),
                          ptr(dev(np.asarray(tokens, np.int32))), ptr(dev(np.asarray(u, np.float32))),
                          ptr(dev(np.asarray(r, np.float32))), ptr(out), ptr(cnt), ptr(err), stream)
    o = host(out, np.int32)
    assert np.all(o[N:] == -7)
    return o[:N], host(cnt, np.int32), int(host(err, np.int32)[0])


def _check_verify(fp, p, q, tokens, u, r, cu):
    B = len(cu) - 1
    out, cnt, err = _verify(fp, p, q, tokens, u, r, cu, B)
    own, fine = np.zeros(len(p), bool), True
    for b in range(B):
        s = slice(cu[b], cu[b + 1])
        own[s] = True
        if cu[b + 1] <= cu[b]:
            assert cnt[b] == 0
            continue
        want, ok = chunk.verify(p[s], None if q is None else q[s], tokens[s], u[s], r[b])
        fine &= ok
        assert cnt[b] == len(want), b
        assert out[s].tolist() == want + [-1] * (cu[b + 1] - cu[b] - len(want)), b
    assert np.all(out[~own] == -7)
    assert err == (0 if fine else 1)
    return out, cnt


def _random_case(rng, V, ks, onehot, sharp, near):
    cu = np.concatenate([[0], np.cumsum([k + 1 if k >= 0 else 0 for k in ks])]) + 1
    N = int(cu[-1]) + 2
    x = sharp * rng.standard_normal((N, V))
    p = chunk.probabilities(x).astype(np.float32)
    q = chunk.probabilities(x + near * rng.standard_normal((N, V))).astype(np.float32)
    after = np.array([np.searchsorted(np.cumsum(row.astype(np.float64)), rng.random() * row.sum(dtype=np.float64)) for row in q])
    after = np.minimum(after, V - 1)
    tokens = np.concatenate([[0], after[:-1]]).astype(np.int32)
    return p, None if onehot else q, tokens, rng.random(N, dtype=np.float32), rng.random(len(ks), dtype=np.float32), cu


@pytest.mark.parametrize("onehot", [False, True])
@pytest.mark.parametrize("V", [1, 2, 5, 127, 128, 129, 1000, 4099, 32000, 70001])
def test_verify(fp, V, onehot):
    rng = np.random.default_rng(V + onehot)
    for sharp, near in ((2.0, 0.5), (0.3, 1.0), (5.0, 0.1)):
        _check_verify(fp, *_random_case(rng, V, [4, 0, -1, 1, 7, 2, 40, 3], onehot, sharp, near))


def test_verify_long_rows(fp):
    rng = np.random.default_rng(5)
    _check_verify(fp, *_random_case(rng, 300007, [2, 0], False, 1.0, 0.7))


def test_verify_borders(fp):
    """Dyadic weights, whose sums are exact: a border that is met belongs to the next token; r = 0 and r >= 1."""
    V = 1024
    p = np.zeros((7, V), np.float32)
    p[:, ::2] = 1.0 / 512  # tokens 0, 2, ..
    r = np.array([0.0, 1 / 512, 1 / 512 - 2.0 ** -30, 0.5, 1 - 2.0 ** -24, 1.0, 1.5], np.float32)
    cu = np.arange(8)
    out, cnt = _check_verify(fp, p, None, np.zeros(7, np.int32), np.zeros(7, np.float32), r, cu)
    assert out.tolist() == [0, 2, 0, 512, 1022, 1022, 1022]


def test_verify_many_draws_on_a_flat_row(fp):
    """1000 borders over a row whose weights are all near 2^-17: each has to fall where fp64 puts it."""
    V, B = 128001, 1000
    rng = np.random.default_rng(9)
    row = (rng.uniform(0.5, 1.5, V) / V).astype(np.float32)
    torch = torch_mod()
    p = torch.from_numpy(row).cuda().repeat(B, 1)
    r = rng.random(B, dtype=np.float32)
    out, cnt, err = empty(B, np.int32), empty(B, np.int32), empty(1, np.int32)
    z = dev(np.zeros(B, np.int32))
    fp.fp_op_verify_draft(ptr(p), None, V, B, B, ptr(dev(np.arange(B + 1, dtype=np.int32))), ptr(z), ptr(z), ptr(dev(r)),
                          ptr(out), ptr(cnt), ptr(err))
    c = np.cumsum(row.astype(np.float64))
    # pairs of fp32 hold a sum to 2^-46 or better: a border nearer than 2^-44 to a token's edge is not judged
    border = r.astype(np.float64) * c[-1]
    want = np.searchsorted(c, border, side="right")
    gap = np.minimum(np.abs(c[want] - border), np.abs(c[np.maximum(want - 1, 0)] - border))
    sure = gap > 2.0 ** -44
    assert sure.sum() > 990
    assert np.array_equal(host(out, np.int32)[sure], want[sure]) and host(err, np.int32)[0] == 0


def test_verify_special_rows(fp):
    V = 300
    rng = np.random.default_rng(7)
    base = chunk.probabilities(rng.standard_normal((2, V))).astype(np.float32)
    p, q = base.copy(), (2 * base).astype(np.float32)
    # q covers p everywhere: nothing is left of the difference, the target itself is drawn from
    _check_verify(fp, p, q, np.array([0, 5], np.int32), np.array([0.9, 0], np.float32), np.array([0.37], np.float32), [0, 2])
    # a token of probability zero is refused whatever u, one of a q of zero accepted
    p2, q2 = base.copy(), base.copy()
    p2[0, 5] = 0
    _check_verify(fp, p2, q2, np.array([0, 5]), np.array([0.0, 0], np.float32), np.array([0.5], np.float32), [0, 2])
    q2[0, 6] = 0
    _check_verify(fp, p2, q2, np.array([0, 6]), np.array([0.99, 0], np.float32), np.array([0.5], np.float32), [0, 2])
    # a draft outside the vocabulary: refused, reported
    for t in (-1, V, 2 ** 31 - 1):
        _check_verify(fp, base, None, np.array([0, t]), np.array([0.0, 0], np.float32), np.array([0.5], np.float32), [0, 2])
    # nothing to draw from: no token, reported; the other sequence as ever
    p3 = np.concatenate([np.zeros((1, V), np.float32), base])
    _check_verify(fp, p3, None, np.array([0, 0, 5]), np.array([0, 0.0, 0], np.float32), np.array([0.5, 0.25], np.float32),
                  [0, 1, 3])
    for bad in (np.inf,):
        p3[0, 7] = bad
        out, cnt, err = _verify(fp, p3, None, [0, 0, 5], [0, 0.0, 0], [0.5, 0.25], [0, 1, 3], 2)
        assert out[0] == -1 and cnt[0] == 0 and err == 1 and cnt[1] > 0
    # NaN weighs nothing
    p3[0] = base[0]
    p3[0, 7] = np.nan
    ref = p3.copy()
    ref[0, 7] = 0
    out, cnt, err = _verify(fp, p3, None, [0, 0, 5], [0, 0.0, 0], [0.5, 0.25], [0, 1, 3], 2)
    assert err == 0 and out[0] == chunk.draw(ref[0].astype(np.float64), 0.5)


def test_verify_bad_cu_stays_inside(fp):
    rng = np.random.default_rng(8)
    p = chunk.probabilities(rng.standard_normal((6, 50))).astype(np.float32)
    tok, u = rng.integers(0, 50, 6).astype(np.int32), rng.random(6, dtype=np.float32)
    for cu in ([0, 3, 99], [-9, 3, 6], [0, 5, 2], [50, 60, 70]):
        out, cnt, err = _verify(fp, p, None, tok, u, [0.3, 0.6], cu, 2)
        assert err == 1 and out.shape == (6,)


# ------------------------------------------------------------------ together
def _head_logits(fp, x, N, d, V, w):
    out = empty((N, V), np.float32)
    need = fp.fp_op_linear_workspace_bytes(0, N, V, d)
    ws = empty(max(need, 16))
    fp.fp_op_linear(0, 3, ptr(x), N, V, d, ptr(w), None, None, None, ptr(out), ptr(ws), need)
    return out


@pytest.mark.parametrize("kvq", [0, 1])
def test_a_drafted_step_equals_decoding_one_by_one(fp, kvq):
    """Append, attention, head, probabilities, verification: greedy requests (T = 0) accept exactly the drafts that
    decoding token by token, through the decode kernels, would have chosen, and draw its next token."""
    hd, H, Hkv, V, B, k = 128, 8, 2, 500, 3, 4
    d, row = H * hd, (H + 2 * Hkv) * hd
    rng = np.random.default_rng(21 + kvq)
    # token -> its fused QKV row; head: attention output -> logits
    emb = dev(synth.uniform_bf16(61, 1, (V, row), -2, 2))
    w = dev(synth.uniform_bf16(62, 1, (V, d), -1, 1))
    T = 400
    pps = T // 16
    pages = B * pps
    table = dev(rng.permutation(pages).reshape(B, pps).astype(np.int32))
    dt = np.int8 if kvq else np.uint16
    lens = np.array([70, 5, 300], np.int32)
    cs = empty(T * hd, np.float32)
    fp.fp_op_rope_table(T, hd, 10000.0, ptr(cs))
    torch = torch_mod()

    def cache():
        pools = [empty((pages, Hkv, 16, hd), dt) for _ in "kv"]
        sc = [empty((pages, Hkv, 16), np.float32) for _ in "kv"]
        return fp.fp_kv_view(kvq, Hkv, hd, 16, pps, pages, ptr(pools[0]), ptr(pools[1]), ptr(sc[0]) if kvq else None,
                             ptr(sc[1]) if kvq else None, ptr(table))

    err = empty(1, np.int32)
    prompts = [rng.integers(0, V, n).astype(np.int32) for n in lens]

    def rows(tokens):
        out = empty((len(tokens), row), np.uint16)
        out.copy_(emb[torch.from_numpy(np.asarray(tokens, np.int64)).cuda()])
        return out

    def take(view, chunks, pos):
        """A ragged chunk through append, attention and head: logits of every row."""
        n = [len(c) for c in chunks]
        N, mx = sum(n), max(n)
        cu, ps = dev(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)), dev(np.asarray(pos, np.int32))
        x = rows(np.concatenate(chunks))
        fp.fp_op_rope_kv_chunk(ptr(x), row, N, B, H, view, ptr(cu), ptr(ps), ptr(cs), ptr(x), row, ptr(err))
        need = fp.fp_op_attention_chunk_workspace_bytes(B, H, Hkv, hd, mx)
        ws, out = empty(need + 256), empty((N, d), np.uint16)
        fp.fp_op_attention_chunk(ptr(x), row, N, B, H, view, ptr(cu), ptr(ps), mx, T, ptr(out),
                                 (ptr(ws) + 255) // 256 * 256, need, ptr(err))
        return _head_logits(fp, out, N, d, V, w), cu, N

    # the prompts in two pieces each; then one token at a time through the decode kernels
    one = cache()
    take(one, [p[: len(p) // 2] for p in prompts], [0] * B)
    lg, _, N = take(one, [p[len(p) // 2:] for p in prompts], [len(p) // 2 for p in prompts])
    last = np.cumsum([len(p) - len(p) // 2 for p in prompts]) - 1
    nxt = host(lg, np.float32).reshape(N, V)[last].argmax(-1)
    start = nxt.copy()
    greedy, sure = [[] for _ in range(B)], [0] * B
    pos = lens.copy()
    for _ in range(k + 1):
        x = rows(nxt)
        fp.fp_op_rope_kv(ptr(x), B, 1, row, H, one, ptr(dev(pos)), ptr(cs), ptr(err))
        need = fp.fp_op_attention_decode_workspace_bytes(B, H, hd, T)
        ws, out = empty(need), empty((B, d), np.uint16)
        fp.fp_op_attention_decode(ptr(x), row, B, H, one, ptr(dev(pos + 1)), T, ptr(out), ptr(ws), need, ptr(err))
        lg = host(_head_logits(fp, out, B, d, V, w), np.float32).reshape(B, V)
        top = np.sort(lg, -1)
        # the two paths' logits differ by about 2^-8 of their spread: a choice nearer than eight of those may turn
        tie = top[:, -1] - top[:, -2] < 2.0 ** -5 * lg.std(-1)
        nxt = lg.argmax(-1)
        for b in range(B):
            sure[b] += sure[b] == len(greedy[b]) and not tie[b]
            greedy[b].append(int(nxt[b]))
        pos = pos + 1
    # the same prompts, then the start token and k drafts at once; sequence b's draft b + 1 is wrong
    two = cache()
    take(two, [p[: len(p) // 2] for p in prompts], [0] * B)
    take(two, [p[len(p) // 2:] for p in prompts], [len(p) // 2 for p in prompts])
    drafts = [[int(start[b])] + greedy[b][:k] for b in range(B)]
    for b in range(B):
        drafts[b][b + 2 if b + 2 <= k else k] += 1
        drafts[b][b + 2 if b + 2 <= k else k] %= V
    lg, cu, N = take(two, [np.array(x, np.int32) for x in drafts], lens)
    probs = empty((N, V), np.float32)
    fp.fp_op_softmax(ptr(lg), N, V, ptr(empty(N, np.float32)), ptr(probs), ptr(err))
    tok, u, r = dev(np.concatenate(drafts).astype(np.int32)), dev(rng.random(N, dtype=np.float32)), dev(rng.random(B, dtype=np.float32))
    out, cnt = empty(N, np.int32), empty(B, np.int32)
    fp.fp_op_verify_draft(ptr(probs), None, V, N, B, ptr(cu), ptr(tok), ptr(u), ptr(r), ptr(out), ptr(cnt), ptr(err))
    out, cnt = host(out, np.int32).reshape(B, k + 1), host(cnt, np.int32)
    for b in range(B):
        a = b + 1  # accepted before the wrong one
        m = min(a + 1, sure[b])
        assert out[b, :m].tolist() == greedy[b][:m] and (m <= a or cnt[b] == a + 1), (b, out[b], greedy[b], sure)
    assert sum(sure) >= B  # how many choices are no near ties is the inputs' affair: some are
    assert host(err, np.int32)[0] == 0
    assert M is not None and quant is not None


def test_the_whole_step_in_one_graph(fp):
    """Append to verification captured once, replayed with other tokens: the results of calls one by one."""
    torch = torch_mod()
    hd, H, Hkv, V, B, N, T = 128, 8, 2, 1000, 2, 8, 160
    d, row, pps = H * hd, (H + 2 * Hkv) * hd, T // 16
    rng = np.random.default_rng(3)
    table = dev(np.arange(B * pps, dtype=np.int32).reshape(B, pps))
    pools = [dev(synth.uniform_bf16(3, i, (B * pps, Hkv, 16, hd), -1, 1)) for i in (1, 2)]
    view = fp.fp_kv_view(0, Hkv, hd, 16, pps, B * pps, ptr(pools[0]), ptr(pools[1]), None, None, ptr(table))
    cs, err = empty(T * hd, np.float32), empty(1, np.int32)
    fp.fp_op_rope_table(T, hd, 10000.0, ptr(cs))
    w = dev(synth.uniform_bf16(3, 5, (V, d), -1, 1))
    qkv, q, o = empty((N, row), np.uint16), empty((N, d), np.uint16), empty((N, d), np.uint16)
    lg, pr = empty((N, V), np.float32), empty((N, V), np.float32)
    cu, pos, tok = empty(B + 1, np.int32), empty(B, np.int32), empty(N, np.int32)
    u, r, out, cnt = empty(N, np.float32), empty(B, np.float32), empty(N, np.int32), empty(B, np.int32)
    need = fp.fp_op_attention_chunk_workspace_bytes(B, H, Hkv, hd, 6)
    ws = empty(need + 256)
    lin = fp.fp_op_linear_workspace_bytes(0, N, V, d)
    lws = empty(max(lin, 16))
    st = torch.cuda.Stream()
    s = st.cuda_stream

    def step():
        fp.fp_op_rope_kv_chunk(ptr(qkv), row, N, B, H, view, ptr(cu), ptr(pos), ptr(cs), ptr(q), d, ptr(err), s)
        fp.fp_op_attention_chunk(ptr(q), d, N, B, H, view, ptr(cu), ptr(pos), 6, T, ptr(o), (ptr(ws) + 255) // 256 * 256,
                                 need, ptr(err), s)
        fp.fp_op_linear(0, 3, ptr(o), N, V, d, ptr(w), None, None, None, ptr(lg), ptr(lws), lin, s)
        fp.fp_op_softmax(ptr(lg), N, V, None, ptr(pr), ptr(err), s)
        fp.fp_op_verify_draft(ptr(pr), None, V, N, B, ptr(cu), ptr(tok), ptr(u), ptr(r), ptr(out), ptr(cnt), ptr(err), s)

    def fill(seqs, seed):
        x = synth.uniform_bf16(seed, 1, (N, row), -2, 2)
        qkv.copy_(torch.from_numpy(x.view(np.int16)))
        cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum([a for a, _ in seqs])]).astype(np.int32)))
        pos.copy_(torch.from_numpy(np.array([b for _, b in seqs], np.int32)))
        g = np.random.default_rng(seed)
        tok.copy_(torch.from_numpy(g.integers(0, V, N).astype(np.int32)))
        u.copy_(torch.from_numpy((g.random(N) * 0.002).astype(np.float32)))
        r.copy_(torch.from_numpy(g.random(B).astype(np.float32)))
        out.fill_(-7)
        torch.cuda.synchronize()

    fill([(3, 20), (5, 9)], 1)
    with torch.cuda.stream(st):
        step()
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step()
    for seqs, seed in (([(3, 20), (5, 9)], 1), ([(1, 100), (6, 0)], 2), ([(0, 4), (4, 140)], 3)):
        fill(seqs, seed)
        g.replay()
        torch.cuda.synchronize()
        got = host(out, np.int32).copy(), host(cnt, np.int32).copy(), host(pr, np.float32).copy()
        n = sum(a for a, _ in seqs)
        fill(seqs, seed)
        step()
        torch.cuda.synchronize()
        assert np.array_equal(got[0], host(out, np.int32)) and np.array_equal(got[1], host(cnt, np.int32))
        assert np.array_equal(got[2][:n], host(pr, np.float32).reshape(N, V)[:n])
        c, p = np.concatenate([[0], np.cumsum([a for a, _ in seqs])]), host(pr, np.float32).reshape(N, V)
        for b in range(B):
            if seqs[b][0]:
                want, ok = chunk.verify(p[c[b]:c[b + 1]], None, host(tok, np.int32)[c[b]:c[b + 1]],
                                        host(u, np.float32)[c[b]:c[b + 1]], host(r, np.float32)[b])
                assert ok and got[0][c[b]:c[b] + got[1][b]].tolist() == want
    assert rng is not None and host(err, np.int32)[0] == 0
