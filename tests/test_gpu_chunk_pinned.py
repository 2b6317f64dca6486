"""Chunked serving, pinned further: the int8 codes and scales of appended keys bit for bit, small queries against large
key scales, and a drafted step in which every choice counts."""
import numpy as np
import pytest

import synth
from oracle import quant
from tests.gpu_helpers import dev, empty, host, ptr, torch_mod
from tests.test_gpu_chunk import Batch, _append

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp():
    torch_mod()
    import paper_2501_13111_gb300 as fp

    return fp


@pytest.mark.parametrize("hd,H,Hkv", [(64, 8, 8), (128, 8, 1), (128, 64, 8), (128, 5, 5)])
def test_appended_int8_keys_bit_for_bit(fp, hd, H, Hkv):
    """What an int8 cache holds of a key is the quantiser's codes and scale of the rotated key that a bf16 cache holds."""
    seqs = [(3, 0), (0, 5), (40, 9), (1, 150), (17, 16)]
    caches = [Batch(fp, kvq, hd, H, Hkv, seqs, 121, lead=2, tail=3) for kvq in (0, 1)]
    c, d = caches
    qkv = synth.uniform_bf16(122, hd, (c.N, (H + 2 * Hkv) * hd), -3, 3)
    qkv[5, H * hd:(H + 1) * hd] = 0  # a key of zeros
    outs = [_append(x, qkv) for x in caches]
    assert outs[0][3] == outs[1][3] == 0
    assert np.array_equal(outs[0][0], outs[1][0])  # the queries
    k16 = host(c.dev["k"], np.uint16).reshape(c.data["k"].shape)
    k8, ks = host(d.dev["k"], np.int8).reshape(d.data["k"].shape), host(d.dev["ks"], np.float32).reshape(d.data["ks"].shape)
    for b, (n, p) in enumerate(seqs):
        if n == 0:
            continue
        at = p + np.arange(n)
        codes, scales = quant.quantize_kv_int8(k16[c.table[b, at // 16], :, at % 16])
        page = d.table[b, at // 16]
        assert np.array_equal(k8[page, :, at % 16], codes) and np.array_equal(ks[page, :, at % 16], scales)
        r = slice(int(d.cu[b]), int(d.cu[b]) + n)
        assert np.array_equal(outs[1][1][r, : Hkv * hd].reshape(n, Hkv, hd),
                              synth.f32_to_bf16_bits(codes.astype(np.float32) * scales[..., None]))


@pytest.mark.parametrize("times", [1e-6, 1e6])
def test_attention_int8_key_scales_far_from_one(fp, times):
    """Queries of 2e6 against key scales of 1e-8, and of 2e-6 against scales of 1e4."""
    c = Batch(fp, 1, 128, 4, 2, [(4, 60), (20, 300)], 123)
    c.data["ks"] = (c.data["ks"] * times).astype(np.float32)
    c.dev["ks"] = dev(c.data["ks"])
    c.view = c.make_view(c.table)
    q = c.queries(8, scale=2 / times)
    got, err = c.attend(q)
    assert err == 0
    c.check(q, got)


@pytest.mark.parametrize("kvq", [0, 1])
def test_a_drafted_step_accepts_what_decoding_would_choose(fp, kvq):
    """Append, attention, head, probabilities, verification at T = 0 against decoding token by token through the decode
    kernels.  The head is the first of a list of seeds with which none of decoding's choices is a near tie, so that
    every sequence's count and every token is compared."""
    torch = torch_mod()
    hd, H, Hkv, V, B, k, T = 128, 8, 2, 300, 3, 4, 400
    d, row, pps = H * hd, (H + 2 * Hkv) * hd, T // 16
    rng = np.random.default_rng(31 + kvq)
    emb = dev(synth.uniform_bf16(131, 1, (V, row), -2, 2))
    pages = B * pps
    table = dev(rng.permutation(pages).reshape(B, pps).astype(np.int32))
    lens = np.array([70, 5, 300], np.int32)
    prompts = [rng.integers(0, V, n).astype(np.int32) for n in lens]
    cs, err = empty(T * hd, np.float32), empty(1, np.int32)
    fp.fp_op_rope_table(T, hd, 10000.0, ptr(cs))
    lin = fp.fp_op_linear_workspace_bytes(0, B * (k + 1), V, d)
    lws = empty(max(lin, 16))

    def cache():
        pools = [empty((pages, Hkv, 16, hd), np.int8 if kvq else np.uint16) for _ in "kv"]
        sc = [ptr(empty((pages, Hkv, 16), np.float32)) if kvq else None for _ in "kv"]
        return fp.fp_kv_view(kvq, Hkv, hd, 16, pps, pages, ptr(pools[0]), ptr(pools[1]), sc[0], sc[1], ptr(table))

    def rows(tokens):
        return emb[torch.from_numpy(np.asarray(tokens, np.int64)).cuda()].contiguous()

    def head(w, x, n):
        lg = empty((n, V), np.float32)
        fp.fp_op_linear(0, 3, ptr(x), n, V, d, ptr(w), None, None, None, ptr(lg), ptr(lws), lin)
        return lg

    def take(view, chunks, pos):
        """A ragged chunk through append and attention: every row's output."""
        n = [len(c) for c in chunks]
        N, mx = sum(n), max(n)
        cu, ps = dev(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)), dev(np.asarray(pos, np.int32))
        x = rows(np.concatenate(chunks))
        fp.fp_op_rope_kv_chunk(ptr(x), row, N, B, H, view, ptr(cu), ptr(ps), ptr(cs), ptr(x), row, ptr(err))
        need = fp.fp_op_attention_chunk_workspace_bytes(B, H, Hkv, hd, mx)
        ws, out = empty(need + 256), empty((N, d), np.uint16)
        fp.fp_op_attention_chunk(ptr(x), row, N, B, H, view, ptr(cu), ptr(ps), mx, T, ptr(out),
                                 (ptr(ws) + 255) // 256 * 256, need, ptr(err))
        torch.cuda.synchronize()
        return out, cu, N

    def prompted():
        view = cache()
        take(view, [p[: len(p) // 2] for p in prompts], [0] * B)
        take(view, [p[len(p) // 2:] for p in prompts], [len(p) // 2 for p in prompts])
        return view

    start = rng.integers(0, V, B).astype(np.int32)

    def decode(w):
        """Greedy tokens of k + 1 steps, or None at a near tie."""
        view, pos, nxt, out = prompted(), lens.copy(), start.copy(), [[] for _ in range(B)]
        need = fp.fp_op_attention_decode_workspace_bytes(B, H, hd, T)
        ws, o = empty(need), empty((B, d), np.uint16)
        for _ in range(k + 1):
            x = rows(nxt)
            fp.fp_op_rope_kv(ptr(x), B, 1, row, H, view, ptr(dev(pos)), ptr(cs), ptr(err))
            fp.fp_op_attention_decode(ptr(x), row, B, H, view, ptr(dev(pos + 1)), T, ptr(o), ptr(ws), need, ptr(err))
            lg = host(head(w, o, B), np.float32).reshape(B, V)
            top = np.sort(lg, -1)
            # the two paths' logits differ by about 2^-8 of their spread
            if np.any(top[:, -1] - top[:, -2] < 2.0 ** -5 * lg.std(-1)):
                return None
            nxt = lg.argmax(-1).astype(np.int32)
            for b in range(B):
                out[b].append(int(nxt[b]))
            pos = pos + 1
        return out

    for seed in range(200):
        w = dev(synth.uniform_bf16(132, seed, (V, d), -1, 1))
        greedy = decode(w)
        if greedy:
            break
    assert greedy, "no head without near ties"
    # the start token and k drafts at once: sequence 0's first draft is wrong, sequence 1's third, sequence 2's none
    drafts = [[int(start[b])] + greedy[b][:k] for b in range(B)]
    accepted = [0, 2, k]
    for b in range(B):
        if accepted[b] < k:
            drafts[b][accepted[b] + 1] = (drafts[b][accepted[b] + 1] + 1) % V
    o, cu, N = take(prompted(), [np.array(x, np.int32) for x in drafts], lens)
    lg, probs = head(w, o, N), empty((N, V), np.float32)
    fp.fp_op_softmax(ptr(lg), N, V, ptr(empty(N, np.float32)), ptr(probs), ptr(err))
    tok, u, r = dev(np.concatenate(drafts).astype(np.int32)), dev(rng.random(N, dtype=np.float32)), dev(rng.random(B, dtype=np.float32))
    out, cnt = empty(N, np.int32), empty(B, np.int32)
    fp.fp_op_verify_draft(ptr(probs), None, V, N, B, ptr(cu), ptr(tok), ptr(u), ptr(r), ptr(out), ptr(cnt), ptr(err))
    assert host(cnt, np.int32).tolist() == [a + 1 for a in accepted]
    got = host(out, np.int32).reshape(B, k + 1)
    for b, a in enumerate(accepted):
        assert got[b].tolist() == greedy[b][: a + 1] + [-1] * (k - a), b
    assert host(err, np.int32)[0] == 0
