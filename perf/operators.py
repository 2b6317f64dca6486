"""The operators of chunked serving, as cases that can be timed and compared: a chunk of new tokens per sequence (the
next piece of a prompt, or drafted tokens to be checked) against a paged cache.

  kv        fp_op_rope_kv_chunk, then fp_op_kv_read: the chunk's queries rotated, its keys rotated and appended with its
            values to the cache (bf16, or int8 with a scale per token and head), and the new positions read back
  attention fp_op_attention_chunk: the chunk's queries over everything cached up to each of them
  softmax   fp_op_softmax: logits to probabilities, a temperature a row (0: the greedy choice)
  verify    fp_op_verify_draft: drafted tokens accepted or refused against the target's probabilities, and the token
            drawn after the last accepted one, from given random numbers

Batches are ragged: sequence b's new tokens are rows cu[b] .. cu[b+1]-1 and sit at positions pos[b] on.  Shapes are those
of the repository's own workloads (tiny, 7B-, 13B- and 70B-shaped blocks, vocabulary 32000) and odd ones between them.
"""
import math
import random

import torch

own = False

PAGE = 16
ROPE_BASE = 10000.0


def listed():
    return [
        # Drafted tokens of 32 sequences (70B-shaped block, int8 cache): a few rows each, latency and scattered pages.
        {"name": "kv_draft_int8_70b", "kind": "kv", "kvq": 1, "batch": 32, "heads": 64, "kv_heads": 8, "hd": 128,
         "new": 5, "context": 2148},
        # Four prompts taken up in pieces of up to 1000 tokens (13B-shaped block, bf16 cache): streaming.
        {"name": "kv_prompt_bf16_13b", "kind": "kv", "kvq": 0, "batch": 4, "heads": 40, "kv_heads": 40, "hd": 128,
         "new": 1000, "context": 3000},
        # The smallest call: three tokens of one short sequence (tiny block, 64-wide heads).  Latency alone.
        {"name": "attn_few_tiny", "kind": "attention", "kvq": 0, "batch": 1, "heads": 8, "kv_heads": 8, "hd": 64,
         "new": 3, "context": 45},
        # Drafted tokens checked, 7B-shaped block with a key head a query head, contexts to 612: the cache's bytes.
        {"name": "attn_draft_bf16_7b", "kind": "attention", "kvq": 0, "batch": 8, "heads": 32, "kv_heads": 32,
         "hd": 128, "new": 5, "context": 612},
        # Drafted tokens checked, 70B-shaped block, int8 cache, 32 contexts to 2148: the cache's bytes, widened.
        {"name": "attn_draft_int8_70b", "kind": "attention", "kvq": 1, "batch": 32, "heads": 64, "kv_heads": 8,
         "hd": 128, "new": 5, "context": 2148},
        # The next 512 tokens of four prompts, 13B-shaped block: products.
        {"name": "attn_chunk_bf16_13b", "kind": "attention", "kvq": 0, "batch": 4, "heads": 40, "kv_heads": 40,
         "hd": 128, "new": 512, "context": 2048},
        # The next 1024 tokens of two long prompts, 70B-shaped block, int8 cache: the largest, products.
        {"name": "attn_chunk_int8_70b", "kind": "attention", "kvq": 1, "batch": 2, "heads": 64, "kv_heads": 8,
         "hd": 128, "new": 1024, "context": 8000},
        # A mixed batch: one prompt's piece of 400 tokens among 15 sequences that decode one token each.
        {"name": "attn_mixed_bf16_70b", "kind": "attention", "kvq": 0, "batch": 16, "heads": 64, "kv_heads": 8,
         "hd": 128, "new": 400, "context": 2500, "mixed": True},
        # Probabilities of all rows of a verification step: 32 sequences, 5 rows each.
        {"name": "probs_160x32000", "kind": "softmax", "rows": 160, "vocab": 32000},
        # One sequence's rows over a large odd vocabulary: few rows, long ones, none but the first aligned.
        {"name": "probs_3x128001", "kind": "softmax", "rows": 3, "vocab": 128001},
        # Verification of up to 4 drafted tokens of 32 sequences.
        {"name": "verify_32x4", "kind": "verify", "batch": 32, "drafts": 4, "vocab": 32000, "onehot": False},
        # One sequence, up to 7 tokens drafted by a lookup (no draft probabilities), a large odd vocabulary.
        {"name": "verify_lookup_1x7", "kind": "verify", "batch": 1, "drafts": 7, "vocab": 100003, "onehot": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["kv", "attention", "attention", "attention", "softmax", "verify"])
    if kind == "softmax":
        rows = _log(rng, 1, 400)
        return {"kind": kind, "rows": rows, "vocab": _log(rng, 1000, min(200000, 20000000 // rows))}
    if kind == "verify":
        batch = _log(rng, 1, 64)
        return {"kind": kind, "batch": batch, "drafts": rng.randint(0, 8),
                "vocab": _log(rng, 1000, min(200000, 10000000 // batch)), "onehot": rng.random() < 0.3}
    hd = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    c = {"kind": kind, "kvq": rng.randint(0, 1), "batch": _log(rng, 1, 48), "heads": heads, "kv_heads": kv_heads,
         "hd": hd}
    if kind == "kv":
        c["new"] = _log(rng, 1, max(1, 4000 * 80 // (c["batch"] * (heads + 2 * kv_heads))))
        c["context"] = c["new"] + _log(rng, 1, 4000)
        return c
    c["new"] = _log(rng, 1, 1024)
    if rng.random() < 0.3:
        c["mixed"] = True
    # scores of the padded batch: at most those of the largest listed case
    most = 2 * 64 * 1024 * 8000 // (c["batch"] * heads * c["new"])
    if most < 64:
        c["batch"] = max(1, c["batch"] * most // 64)
        most = 2 * 64 * 1024 * 8000 // (c["batch"] * heads * c["new"])
    # and cached keys: at most 1 GB of them in bf16
    most = min(most, (1 << 30) // (c["batch"] * kv_heads * hd * 4), 40000)
    c["context"] = _log(rng, max(1, min(32, most)), max(1, most))
    c["new"] = min(c["new"], c["context"])
    return c


def _lengths(case):
    """(new tokens, position of the first one) of each sequence: by the case alone."""
    r = random.Random("%(batch)d %(new)d %(context)d" % case)
    B, new, T = case["batch"], case["new"], case["context"]
    n, pos = [], []
    for b in range(B):
        if case.get("mixed"):
            k = new if b == B // 2 else 1
        else:
            k = new if b == 0 else r.randint((new + 1) // 2, new)
        end = T if b == 0 else r.randint(max(k, T // 2), T)
        n.append(k)
        pos.append(max(0, end - k))
    return n, pos


def _starts(n):
    cu = [0]
    for k in n:
        cu.append(cu[-1] + k)
    return cu


def _cache(case, g, n, pos, filled):
    """Pools, scales and a shuffled page table that cover every sequence; with the values of its positions, or empty."""
    Hkv, hd, B = case["kv_heads"], case["hd"], case["batch"]
    pps = max((p + k + PAGE - 1) // PAGE for p, k in zip(pos, n)) + 1
    pages = B * pps + 3
    table = torch.randperm(pages, generator=g, device="cuda")[: B * pps].reshape(B, pps).to(torch.int32)
    shape = (pages, Hkv, PAGE, hd)
    c = {"table": table, "pps": pps, "pages": pages}
    for w in "kv":
        x = torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16) if filled else torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        if case["kvq"] == 0:
            c[w] = x
            continue
        x = x.float()
        s = x.abs().amax(-1) / 127
        c[w + "s"] = s
        c[w] = torch.where(s[..., None] > 0, (x / s[..., None]).round(), torch.zeros_like(x)).clamp(-127, 127).to(torch.int8)
    return c


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": case}
    if case["kind"] in ("kv", "attention"):
        n, pos = _lengths(case)
        cu = _starts(n)
        N, B, H, Hkv, hd = cu[-1], case["batch"], case["heads"], case["kv_heads"], case["hd"]
        s.update(N=N, B=B, H=H, Hkv=Hkv, hd=hd, max_new=max(n), max_len=max(p + k for p, k in zip(pos, n)))
        s.update(cu=i32(cu), pos=i32(pos), cache=_cache(case, g, n, pos, case["kind"] == "attention"))
        s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        # the chunk's fused QKV rows, as the projection writes them
        row = (H + 2 * Hkv) * hd
        s["row"] = row
        if case["kind"] == "kv":
            s["qkv"] = torch.randn((N, row), generator=g, device="cuda").to(torch.bfloat16)
            i = torch.arange(hd // 2, dtype=torch.float64, device="cuda")
            a = torch.arange(s["cache"]["pps"] * PAGE, dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (-2 * i / hd)
            s["cs"] = torch.stack([a.cos(), a.sin()], -1).float().contiguous()
            s["q"] = torch.zeros((N, H * hd), dtype=torch.bfloat16, device="cuda")
            s["k"] = torch.zeros((N, Hkv * hd), dtype=torch.bfloat16, device="cuda")
            s["v"] = torch.zeros((N, Hkv * hd), dtype=torch.bfloat16, device="cuda")
        else:
            s["qkv"] = (1.5 * torch.randn((N, row), generator=g, device="cuda")).to(torch.bfloat16)
            s["out"] = torch.zeros((N, H * hd), dtype=torch.bfloat16, device="cuda")
        if own:
            import paper_2501_13111_gb300 as fp

            c = s["cache"]
            p = lambda w: c[w].data_ptr() if w in c else None  # noqa: E731
            s["view"] = fp.fp_kv_view(case["kvq"], Hkv, hd, PAGE, c["pps"], c["pages"], p("k"), p("v"), p("ks"), p("vs"), p("table"))
            if case["kind"] == "attention":
                s["ws_bytes"] = fp.fp_op_attention_chunk_workspace_bytes(B, H, Hkv, hd, s["max_new"])
                s["ws"] = torch.zeros(s["ws_bytes"], dtype=torch.uint8, device="cuda")
        return s
    V = case["vocab"]
    s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if case["kind"] == "softmax":
        M = case["rows"]
        s["logits"] = 3 * torch.randn((M, V), generator=g, device="cuda")
        s["logits"][:, 7::97] = -math.inf  # tokens that a request has banned
        t = 0.5 + torch.rand(M, generator=g, device="cuda")
        s["temp"] = torch.where(torch.arange(M, device="cuda") % 8 == 5, torch.zeros_like(t), t)  # some requests are greedy
        s["probs"] = torch.zeros((M, V), device="cuda")
        return s
    # verify: rows cu[b] .. cu[b+1]-1 are the last accepted token and the drafted ones after it
    B, k = case["batch"], case["drafts"]
    r = random.Random("%d %d %d" % (B, k, V))
    n = [1 + (k if b == 0 else r.randint((k + 1) // 2, k)) for b in range(B)]
    cu = _starts(n)
    N = cu[-1]
    logits = 2.5 * torch.randn((N, V), generator=g, device="cuda")
    s["p"] = torch.softmax(logits, -1)
    q = torch.softmax(logits + torch.randn((N, V), generator=g, device="cuda"), -1)
    after = torch.multinomial(q, 1, generator=g)[:, 0].to(torch.int32)  # drafted after row i
    if case["onehot"]:
        after = torch.where(torch.rand(N, generator=g, device="cuda") < 0.6, s["p"].argmax(-1).to(torch.int32), after)
    s["tokens"] = torch.cat([after.new_zeros(1), after[:-1]])
    s["q"] = None if case["onehot"] else q
    s["u"] = torch.rand(N, generator=g, device="cuda")
    s["r"] = torch.rand(B, generator=g, device="cuda")
    s.update(N=N, B=B, V=V, cu=i32(cu), out=torch.full((N,), -1, dtype=torch.int32, device="cuda"),
             n_out=torch.zeros(B, dtype=torch.int32, device="cuda"))
    return s


# ------------------------------------------------------------------ plain forms
def _rows(s):
    """Sequence and place in its chunk of every row."""
    cu = s["cu"].long()
    t = torch.arange(s["N"], device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, t - cu[b]


def _half(x):
    d = x.shape[-1] // 2
    return x[..., :d], x[..., d:]


def _plain_kv(s):
    c, H, Hkv, hd = s["cache"], s["H"], s["Hkv"], s["hd"]
    b, i = _rows(s)
    at = s["pos"].long()[b] + i
    page, slot = c["table"].long()[b, at // PAGE], at % PAGE
    x = s["qkv"].view(s["N"], H + 2 * Hkv, hd)
    cs = s["cs"][at][:, None]
    lo, hi = _half(x[:, : H + Hkv].float())
    cos, sin = cs[..., 0], cs[..., 1]
    qk = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(torch.bfloat16)
    back = []
    for w, y in (("k", qk[:, H:]), ("v", x[:, H + Hkv :])):
        if s["case"]["kvq"] == 0:
            c[w][page, :, slot] = y
            back.append(c[w][page, :, slot].reshape(s["N"], Hkv * hd))
            continue
        y = y.float()
        sc = y.abs().amax(-1) / 127
        code = torch.where(sc[..., None] > 0, (y / sc[..., None]).round(), torch.zeros_like(y)).clamp(-127, 127)
        c[w][page, :, slot] = code.to(torch.int8)
        c[w + "s"][page, :, slot] = sc
        back.append((c[w][page, :, slot].float() * c[w + "s"][page, :, slot][..., None]).to(torch.bfloat16).reshape(s["N"], Hkv * hd))
    return {"q": qk[:, :H].reshape(s["N"], H * hd), "k": back[0], "v": back[1]}


def _plain_attention(s):
    c, B, H, Hkv, hd, T, n = s["cache"], s["B"], s["H"], s["Hkv"], s["hd"], s["max_len"], s["max_new"]
    G = H // Hkv
    b, i = _rows(s)
    key = torch.arange(T, device="cuda")
    page, slot = c["table"].long()[:, key // PAGE], (key % PAGE)[None]
    kf, vf = c["k"][page, :, slot].float(), c["v"][page, :, slot].float()  # [B, T, Hkv, hd]
    if s["case"]["kvq"]:
        kf = kf * c["ks"][page, :, slot][..., None]
        vf = vf * c["vs"][page, :, slot][..., None]
    q = torch.zeros((B, n, H, hd), device="cuda")  # the ragged chunks side by side
    q[b, i] = s["qkv"][:, : H * hd].float().view(-1, H, hd)
    q = q.view(B, n, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, hd)
    sc = torch.matmul(q, kf.permute(0, 2, 3, 1)).view(B, Hkv, G, n, T)
    sc *= hd ** -0.5
    past = key[None, None] > s["pos"].long()[:, None, None] + torch.arange(n, device="cuda")[None, :, None]
    sc.masked_fill_(past[:, None, None], -math.inf)
    sc -= sc.amax(-1, keepdim=True)
    sc.exp_()
    sc /= sc.sum(-1, keepdim=True)
    o = torch.matmul(sc.view(B, Hkv, G * n, T), vf.permute(0, 2, 1, 3)).view(B, Hkv, G, n, hd)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, H * hd)[b, i].to(torch.bfloat16)


def _plain_softmax(s):
    x, t = s["logits"], s["temp"][:, None]
    greedy = t == 0
    e = ((x - x.amax(-1, keepdim=True)) / torch.where(greedy, torch.ones_like(t), t)).exp()
    one = torch.zeros_like(x).scatter_(1, x.argmax(-1, keepdim=True), 1.0)
    return torch.where(greedy, one, e / e.sum(-1, keepdim=True))


def _plain_verify(s):
    p, q, cu, B, N, V = s["p"], s["q"], s["cu"].long(), s["B"], s["N"], s["V"]
    row = torch.arange(N, device="cuda")
    b, i = _rows(s)
    last = cu[b + 1] - 1
    nxt = s["tokens"].long()[torch.clamp(row + 1, max=N - 1)]  # drafted after row i
    pd = p[row, nxt].double()
    qd = q[row, nxt].double() if q is not None else torch.ones_like(pd)
    refused = (s["u"].double() * qd >= pd) & (row < last)
    # accepted drafts: those before the first refusal
    first = torch.where(refused, i, last - cu[b])
    a = torch.full((B,), N, dtype=torch.long, device="cuda").scatter_reduce_(0, b, first, "amin")
    at = cu[:-1] + a
    w, t = p[at].double(), nxt[at]
    if q is not None:
        rest = (w - q[at].double()).clamp(min=0)
    else:
        rest = w.scatter(1, t[:, None], 0.0)
    inner = at < cu[1:] - 1
    w = torch.where((inner & (rest.sum(-1) > 0))[:, None], rest, w)
    cum = w.cumsum(-1)
    drawn = (cum > s["r"].double()[:, None] * cum[:, -1:]).to(torch.uint8).argmax(-1)
    out = torch.where(i < a[b], nxt, torch.where(i == a[b], drawn[b], torch.full_like(nxt, -1)))
    return {"tokens": out.to(torch.int32), "count": (a + 1).to(torch.int32)}


# ------------------------------------------------------------------ the framework's calls
def _own_kv(s):
    import paper_2501_13111_gb300 as fp

    st = torch.cuda.current_stream().cuda_stream
    args = s["cu"].data_ptr(), s["pos"].data_ptr()
    fp.fp_op_rope_kv_chunk(s["qkv"].data_ptr(), s["row"], s["N"], s["B"], s["H"], s["view"], *args, s["cs"].data_ptr(),
                           s["q"].data_ptr(), s["H"] * s["hd"], s["err"].data_ptr(), st)
    fp.fp_op_kv_read(s["view"], s["N"], s["B"], *args, s["k"].data_ptr(), s["v"].data_ptr(), s["Hkv"] * s["hd"],
                     s["err"].data_ptr(), st)
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def _own_attention(s):
    import paper_2501_13111_gb300 as fp

    fp.fp_op_attention_chunk(s["qkv"].data_ptr(), s["row"], s["N"], s["B"], s["H"], s["view"], s["cu"].data_ptr(),
                             s["pos"].data_ptr(), s["max_new"], s["max_len"], s["out"].data_ptr(), s["ws"].data_ptr(),
                             s["ws_bytes"], s["err"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return s["out"]


def _own_softmax(s):
    import paper_2501_13111_gb300 as fp

    M, V = s["logits"].shape
    fp.fp_op_softmax(s["logits"].data_ptr(), M, V, s["temp"].data_ptr(), s["probs"].data_ptr(), s["err"].data_ptr(),
                     torch.cuda.current_stream().cuda_stream)
    return s["probs"]


def _own_verify(s):
    import paper_2501_13111_gb300 as fp

    q = s["q"].data_ptr() if s["q"] is not None else None
    fp.fp_op_verify_draft(s["p"].data_ptr(), q, s["V"], s["N"], s["B"], s["cu"].data_ptr(), s["tokens"].data_ptr(),
                          s["u"].data_ptr(), s["r"].data_ptr(), s["out"].data_ptr(), s["n_out"].data_ptr(),
                          s["err"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return {"tokens": s["out"], "count": s["n_out"]}


_PLAIN = {"kv": _plain_kv, "attention": _plain_attention, "softmax": _plain_softmax, "verify": _plain_verify}
_OWN = {"kv": _own_kv, "attention": _own_attention, "softmax": _own_softmax, "verify": _own_verify}


def run(state):
    kind = state["case"]["kind"]
    return _OWN[kind](state) if own else _PLAIN[kind](state)


def work(case):
    if case["kind"] == "softmax":
        return {"bytes": 8 * case["rows"] * case["vocab"], "flops": 4 * case["rows"] * case["vocab"]}
    if case["kind"] == "verify":
        # one row of each distribution a sequence: where the first draft is refused (or, the target's alone, none is)
        rows = case["batch"] * (1 if case["onehot"] else 2)
        return {"bytes": 4 * rows * case["vocab"], "flops": 2 * rows * case["vocab"]}
    n, pos = _lengths(case)
    H, Hkv, hd = case["heads"], case["kv_heads"], case["hd"]
    cached = 2 * Hkv * (hd + 4 if case["kvq"] else 2 * hd)  # bytes of a position
    N = sum(n)
    if case["kind"] == "kv":
        return {"bytes": N * (2 * (H + 2 * Hkv) * hd + 2 * H * hd + 2 * cached + 4 * Hkv * hd), "flops": 6 * N * (H + Hkv) * hd}
    pairs = sum(k * p + k * (k + 1) // 2 for p, k in zip(pos, n))
    return {"bytes": N * 4 * H * hd + cached * sum(p + k for p, k in zip(pos, n)), "flops": 4 * pairs * H * hd}


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_seq(s, w, b, length):
    """Cached K or V of sequence b as float64 [Hkv, length, hd]."""
    c = s["cache"]
    x = c[w][c["table"][b].long()].double()  # pages, heads, slots, hd
    if s["case"]["kvq"]:
        x = x * c[w + "s"][c["table"][b].long()].double().unsqueeze(-1)
    return x.transpose(0, 1).flatten(1, 2)[:, :length]


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "softmax":
        rows = []
        for x, t in zip(s["logits"].double(), s["temp"].double().tolist()):
            if t > 0:
                z = x / t
                rows.append((z - torch.logsumexp(z, 0)).exp())
            else:
                one = torch.zeros_like(x)
                one[int((x == x.max()).nonzero()[0])] = 1
                rows.append(one)
        return torch.stack(rows)
    cu = s["cu"].tolist()
    if case["kind"] == "verify":
        import numpy as np

        p, u, r, tok = s["p"].cpu().numpy().astype(np.float64), s["u"].tolist(), s["r"].tolist(), s["tokens"].tolist()
        q = None if s["q"] is None else s["q"].cpu().numpy().astype(np.float64)
        out, count = np.full(s["N"], -1, np.int32), np.zeros(s["B"], np.int32)
        for b in range(s["B"]):
            row, end = cu[b], cu[b + 1] - 1
            while row < end and u[row] * (1.0 if q is None else q[row, tok[row + 1]]) < p[row, tok[row + 1]]:
                out[row] = tok[row + 1]
                row += 1
            w = p[row]
            if row < end:
                rest = p[row].copy()
                if q is None:
                    rest[tok[row + 1]] = 0
                else:
                    rest = np.maximum(rest - q[row], 0)
                w = rest if rest.sum() > 0 else w
            total = np.cumsum(w)
            out[row] = int(np.searchsorted(total, r[b] * total[-1], side="right"))
            count[b] = row - cu[b] + 1
        return {"tokens": torch.from_numpy(out), "count": torch.from_numpy(count)}
    pos, H, Hkv, hd = s["pos"].tolist(), s["H"], s["Hkv"], s["hd"]
    if case["kind"] == "kv":
        at = torch.cat([torch.arange(p, p + e - a) for p, a, e in zip(pos, cu, cu[1:])]).double()
        ang = (at[:, None] * ROPE_BASE ** (-2 * torch.arange(hd // 2).double() / hd)).cuda()[:, None]
        turn = torch.polar(torch.ones_like(ang), ang)
        x = s["qkv"].double().view(s["N"], -1, hd)
        z = torch.complex(x[:, : H + Hkv, : hd // 2], x[:, : H + Hkv, hd // 2 :]) * turn
        qk = torch.cat([z.real, z.imag], -1)
        res = {"q": qk[:, :H].flatten(1)}
        for w, y in (("k", qk[:, H:]), ("v", x[:, H + Hkv :])):
            if case["kvq"]:
                y = y.to(torch.bfloat16).double()  # what is quantised
                m = y.abs().max(-1, keepdim=True).values.clamp(min=1e-300)
                y = torch.round(y / m * 127) * (m / 127)
            res[w] = y.flatten(1)
        return res
    out = torch.zeros((s["N"], H, hd), dtype=torch.float64, device="cuda")
    x = s["qkv"][:, : H * hd].double().view(s["N"], H, hd)
    for b in range(s["B"]):
        L = pos[b] + cu[b + 1] - cu[b]
        k, v = _exact_seq(s, "k", b, L), _exact_seq(s, "v", b, L)
        upto = torch.arange(pos[b] + 1, L + 1, device="cuda")[:, None]
        seen = torch.arange(L, device="cuda")[None] < upto
        for h in range(H):
            z = x[cu[b] : cu[b + 1], h] @ k[h // (H // Hkv)].T / math.sqrt(hd)
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            out[cu[b] : cu[b + 1], h] = torch.softmax(z, -1) @ v[h // (H // Hkv)]
    return out.flatten(1)
