"""Chunks of new tokens over the paged cache against the oracle: append and read back, attention.

Tolerance of the attention, element by element, with u = 2^-8 (bf16's half step): the output's own rounding,
u |o|; the probabilities' rounding before the second product, at most u sum_j p_j |v_j|; scores in fp32 (128 products
of at most 4 with a scale of hd^-1/2) move a probability by less than 2^-10.  An int8 cache's codes are exact in bf16,
its scales multiply in fp32.  So
    |got - o| <= 2^-8 |o| + (2^-8 + 2^-10) sum_j p_j |v_j|.
"""
import numpy as np
import pytest

import synth
from oracle import model as M
from oracle import quant
from tests.gpu_helpers import dev, empty, host, ptr, torch_mod

pytestmark = pytest.mark.gpu

BASE = 10000.0


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


class Batch:
    """A ragged batch: (rows, position of the first) of each sequence, its paged cache filled with seeded values and,
    in every slot that no sequence reaches, with `junk`."""

    def __init__(self, fp, kvq, hd, H, Hkv, seqs, seed, lead=0, tail=0, spare=20, junk=None, scale=2.0, vs=(0.001, 0.03)):
        self.fp, self.kvq, self.hd, self.H, self.Hkv, self.seqs = fp, kvq, hd, H, Hkv, seqs
        n = [s[0] for s in seqs]
        self.cu = (lead + np.concatenate([[0], np.cumsum(n)])).astype(np.int32)
        self.pos = np.array([s[1] for s in seqs], np.int32)
        self.B, self.N = len(seqs), int(self.cu[-1]) + tail
        self.max_new = max(max(n), 1)
        self.max_len = max(max(k + p for k, p in seqs), 1)
        self.pps = (self.max_len + spare + 15) // 16
        self.pages = self.B * self.pps + 2
        rng = np.random.default_rng(seed)
        self.table = rng.permutation(self.pages)[: self.B * self.pps].reshape(self.B, self.pps).astype(np.int32)
        shape = (self.pages, Hkv, 16, hd)
        self.data = {}
        live = np.zeros((self.pages, 16), bool)
        for b, (k, p) in enumerate(seqs):
            t = np.arange(max(0, min(k + p, self.pps * 16)))
            live[self.table[b, t // 16], t % 16] = True
        dead = ~live[:, None, :].repeat(Hkv, 1)
        for i, w in enumerate("kv"):
            if kvq == 0:
                x = synth.uniform_bf16(seed, 1 + i, shape, -scale, scale)
                if junk is not None:
                    x[dead] = synth.f32_to_bf16_bits(np.array([junk], np.float32))[0]
                self.data[w] = x
            else:
                self.data[w] = rng.integers(-127, 128, shape, dtype=np.int8)
                s = synth.uniform_f32(seed, 3 + i, shape[:3], *((0.001, 0.03) if w == "k" else vs))
                if junk is not None:
                    s[dead] = junk
                self.data[w + "s"] = s
        self.dev = {w: dev(x) for w, x in self.data.items()}
        self.view = self.make_view(self.table)

    def make_view(self, table):
        d = self.dev
        return self.fp.fp_kv_view(self.kvq, self.Hkv, self.hd, 16, self.pps, self.pages, ptr(d["k"]), ptr(d["v"]),
                                  ptr(d.get("ks")), ptr(d.get("vs")), ptr(dev(table)))

    def cached(self, w, b, length, table=None):
        """K or V of positions 0 .. length-1 of sequence b as fp64 [length, Hkv, hd]; a bad page: zeros."""
        t = np.arange(length)
        page = (self.table if table is None else table)[b, t // 16]
        bad = (page < 0) | (page >= self.pages)
        page, slot = np.where(bad, 0, page), t % 16
        x = self.data[w][page, :, slot]
        x = quant.bf16_to_f32(x).astype(np.float64) if self.kvq == 0 else \
            x.astype(np.float64) * self.data[w + "s"][page, :, slot].astype(np.float64)[..., None]
        x[bad] = 0.0
        return x

    def queries(self, seed, stride=None, scale=2.0):
        return synth.uniform_bf16(seed, 31, (self.N, stride or self.H * self.hd), -scale, scale)

    def attend(self, q, out=None, view=None, cu=None, pos=None, max_new=None, max_len=None, ws=None, stream=None,
               sync=True):
        f = self.fp
        qd = q if hasattr(q, "data_ptr") else dev(q)
        out = out if out is not None else dev(np.full((self.N, self.H * self.hd), 0x4321, np.uint16))
        need = f.fp_op_attention_chunk_workspace_bytes(self.B, self.H, self.Hkv, self.hd, max_new or self.max_new)
        if ws is None:
            ws = empty(need + 256)
            ws[65536:] = 255  # behind the tickets any content will do
        err = empty(1, np.int32)
        f.fp_op_attention_chunk(ptr(qd), qd.shape[1], self.N, self.B, self.H, view or self.view,
                                ptr(dev(self.cu if cu is None else cu)), ptr(dev(self.pos if pos is None else pos)),
                                max_new or self.max_new, max_len or self.max_len, ptr(out), (ptr(ws) + 255) // 256 * 256,
                                need, ptr(err), stream)
        if not sync:
            return out, err
        return host(out, np.uint16).reshape(self.N, self.H * self.hd), int(host(err, np.int32)[0])

    def check(self, q, got, only=None, table=None, pos=None):
        """Every row of the sequences against the oracle; rows of none untouched."""
        H, hd, g = self.H, self.hd, self.H // self.Hkv
        owned = np.zeros(self.N, bool)
        for b, (n, p) in enumerate(self.seqs):
            r = slice(int(self.cu[b]), int(self.cu[b]) + n)
            owned[r] = True
            if n == 0 or (only is not None and b not in only):
                continue
            p = p if pos is None else int(pos[b])
            k, v = self.cached("k", b, p + n, table), self.cached("v", b, p + n, table)
            x = quant.bf16_to_f32(q[r, : H * hd]).astype(np.float64).reshape(n, H, hd)
            o = quant.bf16_to_f32(got[r]).astype(np.float64).reshape(n, H, hd)
            ref = M.attention(x, p + np.arange(n), k, v)
            mass = M.attention(x, p + np.arange(n), k, np.abs(v))  # sum p |v|
            off = np.abs(o - ref) / (2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -10) * mass + 1e-30)
            assert np.all(np.isfinite(o)) and off.max() <= 1, (b, off.max(), np.argwhere(off == off.max())[:3], g)
        assert np.all(got[~owned] == 0x4321)


HEADS = [(64, 8, 8), (128, 8, 1), (128, 64, 8), (128, 6, 2), (64, 14, 2), (128, 5, 5), (128, 40, 2), (64, 128, 1)]
BATCHES = [
    [(1, 0)],
    [(3, 0), (0, 17), (1, 300), (5, 15), (130, 1), (16, 112)],
    [(1, 126), (2, 126), (3, 126), (2, 127), (1, 128), (17, 240)],
    [(260, 511)],
    [(1, 1000), (1, 3), (5, 257), (4, 900)] * 6,
    [(4, 5000)],
]


@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("hd,H,Hkv", HEADS)
@pytest.mark.parametrize("kvq", [0, 1])
def test_attention(fp, kvq, hd, H, Hkv, batch):
    c = Batch(fp, kvq, hd, H, Hkv, BATCHES[batch], 7 * batch + hd + H, lead=batch % 2 * 3, tail=5)
    q = c.queries(batch)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("kvq,hd,H,Hkv,seqs", [
    (0, 128, 8, 1, [(700, 1300), (1, 1999), (33, 64)]),
    (1, 128, 16, 2, [(513, 1023), (128, 0), (129, 127)]),
    (0, 64, 4, 4, [(1025, 0), (2, 700)]),
    (0, 128, 2, 2, [(900, 77)]),
    (1, 64, 6, 2, [(640, 3000)]),
    (1, 128, 8, 8, [(300, 0), (299, 1)]),
])
def test_attention_long_chunks(fp, kvq, hd, H, Hkv, seqs):
    c = Batch(fp, kvq, hd, H, Hkv, seqs, 5 + len(seqs))
    q = c.queries(2)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("kvq,hd,H,Hkv,seqs", [
    (0, 128, 8, 1, [(4, 30000)]),            # 59 CTAs share a unit of one tile
    (1, 128, 8, 1, [(1, 20000), (2, 7)]),
    (0, 128, 8, 1, [(64, 12000)]),           # two units of two tiles, 60 CTAs each
    (1, 64, 3, 1, [(100, 9000)]),
    (0, 64, 16, 2, [(3, 16000), (1, 15999)]),
])
def test_attention_units_that_many_ctas_share(fp, kvq, hd, H, Hkv, seqs):
    """More parts of a unit than are added at once: groups of them, then the groups; the tickets are left at zero."""
    c = Batch(fp, kvq, hd, H, Hkv, seqs, 61)
    q = c.queries(14)
    ws = empty(fp.fp_op_attention_chunk_workspace_bytes(c.B, H, Hkv, hd, c.max_new) + 256)
    for _ in range(2):
        got, err = c.attend(q, ws=ws)
        assert err == 0
        c.check(q, got)
    off = -ptr(ws) % 256
    assert not host(ws, np.uint8)[off:off + 65536].any()


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_of_no_rows(fp, kvq):
    """Sequences without rows only, in a buffer that has some: nothing is written, nothing reported."""
    c = Batch(fp, kvq, 128, 4, 2, [(0, 5), (0, 0), (0, 70)], 63, tail=6)
    got, err = c.attend(c.queries(15), max_new=3)
    assert err == 0 and np.all(got == 0x4321)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_queries_inside_the_fused_rows(fp, kvq):
    """q read in place from QKV rows (a stride larger than the heads)."""
    c = Batch(fp, kvq, 128, 8, 2, [(5, 60), (40, 0)], 3)
    q = c.queries(4, stride=12 * 128)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
@pytest.mark.parametrize("junk", [np.nan, np.inf, -3e38])
def test_attention_ignores_what_lies_behind_a_sequence(fp, kvq, junk):
    """Slots of a page behind the last cached position, and pages that no sequence owns, may hold anything."""
    for hd, H, Hkv in [(128, 8, 2), (64, 4, 4)]:
        c = Batch(fp, kvq, hd, H, Hkv, [(1, 0), (3, 14), (2, 200), (140, 5)], 11, junk=junk)
        q = c.queries(5)
        got, err = c.attend(q)
        assert err == 0
        c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_peaked_scores(fp, kvq):
    """Scores of hundreds, so that a running maximum moves far and most probabilities vanish: q = 60 times a cached
    key (score 60 |k|^2 / sqrt(hd)) makes that key all that is seen, its value comes out to the output's rounding."""
    c = Batch(fp, kvq, 128, 4, 2, [(6, 700), (3, 130)], 13)
    q = c.queries(6)
    want = {}
    rng = np.random.default_rng(1)
    for b, (n, p) in enumerate(c.seqs):
        k, v = c.cached("k", b, p + n), c.cached("v", b, p + n)
        for i in range(n):
            for h in range(4):
                j = int(rng.integers(0, p + i + 1))
                kk = k[j, h // 2]
                q[c.cu[b] + i, h * 128:(h + 1) * 128] = synth.f32_to_bf16_bits((60 * kk / np.abs(kk).max()).astype(np.float32))
                want[c.cu[b] + i, h] = (b, j)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("slope", [0.2, 2.0, -0.2])
@pytest.mark.parametrize("hd,H,Hkv", [(128, 4, 2), (64, 8, 1)])
@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_scores_that_rise_with_the_position(fp, kvq, hd, H, Hkv, slope):
    """The running maximum moves in every 64 keys (or never again): what was summed before is scaled each time."""
    c = Batch(fp, kvq, hd, H, Hkv, [(6, 700), (200, 300), (1, 63), (3, 127)], 67, tail=3)
    sign = np.where(np.random.default_rng(5).random(hd) < 0.5, -1.0, 1.0)
    for b in range(c.B):
        t = np.arange(c.pps * 16)
        up = (slope * t if slope > 0 else slope * (t - 700)) / np.sqrt(hd)  # score of a query of 1: slope t
        page, slot = c.table[b, t // 16], t % 16
        if kvq:
            c.data["k"][page, :, slot] = np.where(sign < 0, -100, 100)
            c.data["ks"][page, :, slot] = (up / 100)[:, None]
        else:
            c.data["k"][page, :, slot] = synth.f32_to_bf16_bits((up[:, None] * sign).astype(np.float32))[:, None]
    for w in c.data:
        c.dev[w] = dev(c.data[w])
    c.view = c.make_view(c.table)
    q = np.empty((c.N, H, hd), np.float32)
    q[:] = sign * np.array([1.0, 0.5])[np.arange(H) % 2][:, None]
    q = synth.f32_to_bf16_bits(q).reshape(c.N, H * hd)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("vs", [(1e-7, 3e-7), (50.0, 400.0)])
def test_attention_int8_value_scales(fp, vs):
    c = Batch(fp, 1, 128, 8, 2, [(5, 400), (200, 100)], 17, vs=vs)
    q = c.queries(7)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


def test_attention_int8_large_queries_and_scales(fp):
    """Queries beyond fp16's range against keys as small, and the reverse: bf16 operands carry both."""
    c = Batch(fp, 1, 128, 4, 2, [(4, 60)], 19)
    for w in ("ks",):
        c.data[w] = (c.data[w] * 1e-6).astype(np.float32)
        c.dev[w] = dev(c.data[w])
    c.view = c.make_view(c.table)
    q = c.queries(8, scale=2e6)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_bad_page_reads_zeros(fp, kvq):
    c = Batch(fp, kvq, 128, 8, 2, [(3, 200), (150, 30)], 23)
    table = c.table.copy()
    table[0, 5], table[1, 9] = c.pages, -4
    q = c.queries(9)
    got, err = c.attend(q, view=c.make_view(table))
    assert err == 1
    c.check(q, got, table=table)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_rows_without_keys_and_lengths_beyond_the_bounds(fp, kvq):
    """Rows at negative positions have no keys (zeros); keys behind max_len are not read; rows behind max_new stay."""
    c = Batch(fp, kvq, 128, 8, 2, [(6, 40), (9, 64), (2, 30)], 29)
    q = c.queries(10)
    pos = np.array([-3, 64, 30], np.int32)
    got, err = c.attend(q, pos=pos)
    assert err == 1
    assert np.all(got[0:3] & 0x7FFF == 0)
    x = quant.bf16_to_f32(q[3:6]).astype(np.float64).reshape(3, 8, 128)
    ref = M.attention(x, np.arange(3), c.cached("k", 0, 3), c.cached("v", 0, 3))
    o = quant.bf16_to_f32(got[3:6]).reshape(3, 8, 128)
    assert np.abs(o - ref).max() <= 2.0 ** -7 * 4
    c.check(q, got, only={1, 2})
    # max_len 66: rows of sequence 1 see 65, 66, 66, .. keys
    got, err = c.attend(q, max_len=66)
    assert err == 1
    k, v = c.cached("k", 1, 66), c.cached("v", 1, 66)
    x = quant.bf16_to_f32(q[6:15]).astype(np.float64).reshape(9, 8, 128)
    ref = M.attention(x, np.minimum(64 + np.arange(9), 65), k, v)
    o = quant.bf16_to_f32(got[6:15]).reshape(9, 8, 128)
    assert np.abs(o - ref).max() <= 2.0 ** -7 * 4
    c.check(q, got, only={0, 2})
    # max_new 4: the rows behind stay
    got, err = c.attend(q, max_new=4)
    assert err == 1
    assert np.all(got[4:6] == 0x4321) and np.all(got[10:15] == 0x4321)
    c.check(np.where(np.arange(c.N)[:, None] >= 0, q, q), np.where((got == 0x4321), got, got), only={2})


def test_a_bad_cu_is_reported_and_touches_nothing(fp):
    c = Batch(fp, 0, 128, 4, 2, [(4, 20), (5, 30), (3, 10)], 31, tail=4)
    q = c.queries(11)
    for cu in ([0, 4, 9, 40], [-3, 4, 9, 12], [0, 9, 4, 12], [5, 4, 3, 2], [100, 200, 300, 400], [0, 4, 9, 8]):
        got, err = c.attend(q, cu=np.array(cu, np.int32), max_new=40, max_len=c.max_len)
        assert err == 1 and np.all(got == 0x4321), cu


def test_attention_of_many_sequences(fp):
    """More sequences than a warp has lanes, some without rows, in order and with gaps."""
    rng = np.random.default_rng(4)
    seqs = [(int(n), int(p)) for n, p in zip(rng.integers(0, 4, 100), rng.integers(0, 700, 100))]
    for kvq in (0, 1):
        c = Batch(fp, kvq, 64, 4, 2, seqs, 33, lead=1, tail=2)
        q = c.queries(12)
        got, err = c.attend(q)
        assert err == 0
        c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_attention_captured_and_replayed_with_other_lengths(fp, kvq):
    """One captured launch within bounds serves other ragged batches; two graphs may share a workspace in turn."""
    torch = torch_mod()
    a = Batch(fp, kvq, 128, 16, 2, [(5, 700), (1, 90), (3, 33)], 37, tail=60)
    q = a.queries(12)
    qd, out = dev(q), dev(np.full((a.N, a.H * a.hd), 0x4321, np.uint16))
    cu, pos, err = dev(a.cu), dev(a.pos), empty(1, np.int32)
    need = fp.fp_op_attention_chunk_workspace_bytes(a.B, a.H, a.Hkv, a.hd, 40)
    ws = empty(need + 256)
    st = torch.cuda.Stream()

    def call():
        fp.fp_op_attention_chunk(ptr(qd), qd.shape[1], a.N, a.B, a.H, a.view, ptr(cu), ptr(pos), 40, a.max_len, ptr(out),
                                 (ptr(ws) + 255) // 256 * 256, need, ptr(err), st.cuda_stream)

    with torch.cuda.stream(st):
        call()
    st.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            call()
        graphs.append(g)
    for turn, seqs in enumerate([[(5, 700), (1, 90), (3, 33)], [(1, 0), (40, 660), (0, 9)], [(2, 5), (2, 6), (40, 300)]]):
        a.seqs = seqs
        a.cu = np.concatenate([[0], np.cumsum([s[0] for s in seqs])]).astype(np.int32)
        cu.copy_(torch.from_numpy(a.cu))
        pos.copy_(torch.from_numpy(np.array([s[1] for s in seqs], np.int32)))
        out.fill_(0x4321)
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        a.check(q, host(out, np.uint16).reshape(a.N, -1))
    assert host(err, np.int32)[0] == 0


def test_attention_repeats_bit_for_bit(fp):
    """Splits and their sums follow the lengths alone: a second run gives the same bits, on another stream too, and two
    calls at once with a workspace each."""
    torch = torch_mod()
    c = Batch(fp, 1, 128, 64, 8, [(5, 2100), (3, 900), (64, 1200), (1, 4000)], 41)
    qd = dev(c.queries(13))
    first = c.attend(qd)[0]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [c.attend(qd, stream=s.cuda_stream, sync=False)[0] for s in streams]
    torch.cuda.synchronize()
    for o in outs:
        assert np.array_equal(host(o, np.uint16).reshape(first.shape), first)


def test_attention_page_offsets_past_32_bits(fp):
    """A pool of more than 2^32 bytes and elements: pages at its far end."""
    torch = torch_mod()
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    hd, H, Hkv, n, p = 128, 4, 2, 3, 45
    pages = (1 << 32) // (Hkv * 16 * hd) + 64  # more than 2^32 elements, 8.6 GB a pool
    pool = torch.zeros((2, pages, Hkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    table = np.array([[pages - 1, 3, pages - 17]], np.int32)
    k = synth.uniform_bf16(1, 1, (3, Hkv, 16, hd), -2, 2)
    v = synth.uniform_bf16(1, 2, (3, Hkv, 16, hd), -2, 2)
    for w, x in ((0, k), (1, v)):
        for i, pg in enumerate(table[0]):
            pool[w, int(pg)] = torch.from_numpy(x[i].view(np.int16)).view(torch.bfloat16).cuda()
    view = fp.fp_kv_view(0, Hkv, hd, 16, 3, pages, pool[0].data_ptr(), pool[1].data_ptr(), None, None, ptr(dev(table)))
    q = synth.uniform_bf16(1, 3, (n, H * hd), -2, 2)
    cu, pos, err = dev(np.array([0, n], np.int32)), dev(np.array([p], np.int32)), empty(1, np.int32)
    need = fp.fp_op_attention_chunk_workspace_bytes(1, H, Hkv, hd, n)
    ws, out = empty(need + 256), empty((n, H * hd), np.uint16)
    fp.fp_op_attention_chunk(ptr(dev(q)), H * hd, n, 1, H, view, ptr(cu), ptr(pos), n, p + n, ptr(out),
                             (ptr(ws) + 255) // 256 * 256, need, ptr(err))
    got = quant.bf16_to_f32(host(out, np.uint16)).reshape(n, H, hd)
    kk = quant.bf16_to_f32(k).transpose(0, 2, 1, 3).reshape(48, Hkv, hd).astype(np.float64)
    vv = quant.bf16_to_f32(v).transpose(0, 2, 1, 3).reshape(48, Hkv, hd).astype(np.float64)
    ref = M.attention(quant.bf16_to_f32(q).astype(np.float64).reshape(n, H, hd), p + np.arange(n), kk, vv)
    assert np.abs(got - ref).max() <= 2.0 ** -7 * 2 and host(err, np.int32)[0] == 0
    rk, rv = empty((n, Hkv * hd), np.uint16), empty((n, Hkv * hd), np.uint16)
    fp.fp_op_kv_read(view, n, 1, ptr(cu), ptr(pos), ptr(rk), ptr(rv), Hkv * hd, ptr(err))
    assert np.array_equal(quant.bf16_to_f32(host(rk, np.uint16)).reshape(n, Hkv, hd), kk[p:p + n])
    assert np.array_equal(quant.bf16_to_f32(host(rv, np.uint16)).reshape(n, Hkv, hd), vv[p:p + n])


# ------------------------------------------------------------------ append and read back
def _append(c, qkv, in_place=False, view=None, pos=None, cu=None):
    """fp_op_rope_kv_chunk, then fp_op_kv_read: (q, k, v, err)."""
    f, H, Hkv, hd = c.fp, c.H, c.Hkv, c.hd
    cs = empty(c.pps * 16 * hd, np.float32)
    f.fp_op_rope_table(c.pps * 16, hd, BASE, ptr(cs))
    x = dev(qkv)
    q = x if in_place else dev(np.full((c.N, H * hd + 8), 0x4321, np.uint16))
    k, v = (dev(np.full((c.N, Hkv * hd + 16), 0x4321, np.uint16)) for _ in "kv")
    err = empty(1, np.int32)
    cu, pos = dev(c.cu if cu is None else cu), dev(c.pos if pos is None else pos)
    f.fp_op_rope_kv_chunk(ptr(x), x.shape[1], c.N, c.B, H, view or c.view, ptr(cu), ptr(pos), ptr(cs), ptr(q), q.shape[1],
                          ptr(err))
    f.fp_op_kv_read(view or c.view, c.N, c.B, ptr(cu), ptr(pos), ptr(k), ptr(v), k.shape[1], ptr(err))
    return tuple(host(t, np.uint16).reshape(c.N, -1) for t in (q, k, v)) + (int(host(err, np.int32)[0]),)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("hd,H,Hkv", [(64, 8, 8), (128, 8, 1), (128, 64, 8), (128, 5, 5), (64, 6, 2)])
@pytest.mark.parametrize("kvq", [0, 1])
def test_append_and_read_back(fp, kvq, hd, H, Hkv, in_place):
    """Rotations against fp64 (fp32 products and one bf16 rounding: 2^-8 of the value and 2^-22 of the pair), values
    and their codes bit for bit; everything else in the pools and the outputs as it was."""
    c = Batch(fp, kvq, hd, H, Hkv, [(3, 0), (0, 5), (40, 9), (1, 150), (17, 16)], 43 + hd, lead=2, tail=3)
    qkv = synth.uniform_bf16(44, hd, (c.N, (H + 2 * Hkv) * hd + 8), -3, 3)
    q, k, v, err = _append(c, qkv, in_place)
    assert err == 0
    own = np.zeros(c.N, bool)
    live = np.zeros((c.pages, 16), bool)
    for b, (n, p) in enumerate(c.seqs):
        r, at = slice(int(c.cu[b]), int(c.cu[b]) + n), p + np.arange(n)
        own[r] = True
        live[c.table[b, at // 16], at % 16] = True
        x = qkv[r, : (H + 2 * Hkv) * hd].reshape(n, H + 2 * Hkv, hd)
        f = quant.bf16_to_f32(x).astype(np.float64)
        ref = M.rope(f[:, : H + Hkv], at, BASE)
        size = np.sqrt(f[:, : H + Hkv, : hd // 2] ** 2 + f[:, : H + Hkv, hd // 2:] ** 2)
        # the table holds fp32 cosines of the fp64 angle: 2^-24 of the pair, and three roundings of fp32
        tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -22 * np.concatenate([size, size], -1)
        qg = quant.bf16_to_f32(q[r, : H * hd]).reshape(n, H, hd)
        assert np.all(np.abs(qg - ref[:, :H]) <= tol[:, :H])
        kg = quant.bf16_to_f32(k[r, : Hkv * hd]).reshape(n, Hkv, hd)
        if kvq == 0:
            assert np.all(np.abs(kg - ref[:, H:]) <= tol[:, H:])
            assert np.array_equal(v[r, : Hkv * hd].reshape(n, Hkv, hd), x[:, H + Hkv:])
        else:
            # half a step of the row's scale, and the roundings of K before and of q s after it
            s = np.abs(kg).max(-1, keepdims=True) / 127 if n else 0
            assert np.all(np.abs(kg - ref[:, H:]) <= tol[:, H:] + 0.52 * s + 2.0 ** -8 * np.abs(kg) + 2.0 ** -8 * s * 127 / 2)
            vq, vs = quant.quantize_kv_int8(x[:, H + Hkv:])
            assert np.array_equal(v[r, : Hkv * hd].reshape(n, Hkv, hd),
                                  synth.f32_to_bf16_bits((vq.astype(np.float32) * vs[..., None])))
            pg = c.table[b, at // 16]
            assert np.array_equal(host(c.dev["v"], np.int8).reshape(c.data["v"].shape)[pg, :, at % 16], vq)
            assert np.array_equal(host(c.dev["vs"], np.float32).reshape(c.data["vs"].shape)[pg, :, at % 16], vs)
    assert np.all(k[~own] == 0x4321) and np.all(v[~own] == 0x4321)
    assert np.all(k[:, Hkv * hd:] == 0x4321) and np.all(v[:, Hkv * hd:] == 0x4321)
    if in_place:
        assert np.array_equal(q[~own], qkv[~own]) and np.array_equal(q[:, H * hd:], qkv[:, H * hd:])
    else:
        assert np.all(q[~own] == 0x4321) and np.all(q[:, H * hd:] == 0x4321)
    for w in "kv":
        after = host(c.dev[w], c.data[w].dtype).reshape(c.data[w].shape)
        rest = ~live[:, None, :].repeat(Hkv, 1)
        assert np.array_equal(after[rest], c.data[w][rest])


@pytest.mark.parametrize("kvq", [0, 1])
def test_append_equals_the_uniform_append(fp, kvq):
    """A batch of equal chunks gives what fp_op_rope_kv gives, to a step of bf16 where the two orders of a rotation
    round apart (an int8 code then moves by one)."""
    c = Batch(fp, kvq, 128, 4, 2, [(5, 0), (5, 9), (5, 30)], 47)
    qkv = synth.uniform_bf16(48, 1, (c.N, 8 * 128), -3, 3)
    q, k, v, err = _append(c, qkv)
    d = Batch(fp, kvq, 128, 4, 2, [(5, 0), (5, 9), (5, 30)], 47)
    cs = empty(d.pps * 16 * 128, np.float32)
    fp.fp_op_rope_table(d.pps * 16, 128, BASE, ptr(cs))
    x, e = dev(qkv), empty(1, np.int32)
    fp.fp_op_rope_kv(ptr(x), 3, 5, 8 * 128, 4, d.view, ptr(dev(d.pos)), ptr(cs), ptr(e))
    a = quant.bf16_to_f32(q[:, : 4 * 128])
    b = quant.bf16_to_f32(host(x, np.uint16).reshape(c.N, -1)[:, : 4 * 128])
    assert np.all(np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + 2.0 ** -20)
    va, vb = (host(t.dev["v"], t.data["v"].dtype) for t in (c, d))
    assert np.array_equal(va, vb) and err == 0


@pytest.mark.parametrize("kvq", [0, 1])
def test_append_skips_what_has_no_place(fp, kvq):
    """Positions outside the cache and bad pages: reported, nothing written there, the other rows as ever."""
    c = Batch(fp, kvq, 128, 4, 2, [(4, 40), (4, 20), (4, 30)], 53)
    qkv = synth.uniform_bf16(54, 1, (c.N, 8 * 128), -3, 3)
    good = _append(c, qkv)
    c = Batch(fp, kvq, 128, 4, 2, [(4, 40), (4, 20), (4, 30)], 53)
    q, k, v, err = _append(c, qkv, pos=np.array([c.pps * 16 - 2, -2, 30], np.int32))
    assert err == 1
    assert np.array_equal(q[8:], good[0][8:]) and np.array_equal(k[8:], good[1][8:]) and np.array_equal(v[8:], good[2][8:])
    assert np.all(q[2:4] == 0x4321) and np.all(q[4:6] == 0x4321)
    assert np.all(k[2:6, : 2 * 128] == 0) and np.all(v[2:6, : 2 * 128] == 0)
    c = Batch(fp, kvq, 128, 4, 2, [(4, 40), (4, 20), (4, 30)], 53)
    table = c.table.copy()
    table[1, 1] = c.pages
    q, k, v, err = _append(c, qkv, view=c.make_view(table))
    assert err == 1
    assert np.array_equal(q, good[0])  # queries need no page
    assert np.all(k[4:8, : 2 * 128] == 0) and np.array_equal(k[8:], good[1][8:]) and np.array_equal(k[:4], good[1][:4])
    for cu in ([0, 4, 8, 99], [0, 8, 4, 12], [-5, 4, 8, 12]):
        c = Batch(fp, kvq, 128, 4, 2, [(4, 40), (4, 20), (4, 30)], 53)
        assert _append(c, qkv, cu=np.array(cu, np.int32))[3] == 1


def test_int8_rows_of_zeros_and_extremes(fp):
    """A row of zeros has scale 0 and reads back as zeros; the largest bf16 keeps its row finite."""
    c = Batch(fp, 1, 64, 2, 1, [(3, 0)], 59)
    x = np.zeros((3, 4 * 64), np.float32)
    x[1] = 3.0e38
    x[2, 192:] = np.linspace(-1e-30, 1e-30, 64)
    q, k, v, err = _append(c, synth.f32_to_bf16_bits(x))
    assert err == 0
    assert np.all(v[0, :64] == 0) and np.all(k[0, :64] == 0)
    vf = quant.bf16_to_f32(v[1, :64])
    assert np.all(np.abs(vf / 3.0e38 - 1) <= 2.0 ** -7)
    vq, vs = quant.quantize_kv_int8(synth.f32_to_bf16_bits(x)[2, 192:][None])
    assert np.array_equal(v[2, :64], synth.f32_to_bf16_bits(vq[0].astype(np.float32) * vs[0]))
