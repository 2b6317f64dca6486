"""The operators for several continuations of a sequence over one paged cache, as cases that can be timed and compared:
trees of drafted tokens, and beams.

  cache     fp_op_tree_plan, fp_op_rope_kv_tree, fp_op_kv_commit: depths and ancestor masks of the drafted trees, their
            queries and keys rotated by depth and appended row by row, then the rows of an accepted path moved together
            (and fp_op_kv_read, to look at what the cache holds now)
  attention fp_op_attention_tree: each drafted row over the cached prefix and its own ancestors
  verify    fp_op_verify_tree: a token drawn after each accepted row, the row's child with that token accepted next
  select    fp_op_beam_select: the best continuations of each group of beams over beams and vocabulary
  reorder   fp_op_beam_reorder, fp_op_kv_copy: page tables that follow the chosen beams, part-filled pages copied
            (and fp_op_kv_read)

Batches are ragged: sequence b's rows are cu[b] .. cu[b+1]-1 and stand at cache positions pos[b] on; row 0 is the last
accepted token, the root of its tree.  Shapes are those of the repository's own workloads (tiny, 7B-, 13B- and 70B-shaped
blocks, vocabulary 32000) and odd ones between them.
"""
import math
import random

import torch

own = False

PAGE = 16
ROPE_BASE = 10000.0


def listed():
    return [
        # One layer's cache work of a verification step: 32 trees of up to 16 rows, 70B-shaped block, int8 cache.
        {"name": "cache_int8_70b", "kind": "cache", "kvq": 1, "batch": 32, "heads": 64, "kv_heads": 8, "hd": 128,
         "nodes": 16, "context": 2148},
        # The same for eight large trees with a key head a query head (13B-shaped block, bf16 cache): bytes.
        {"name": "cache_bf16_13b", "kind": "cache", "kvq": 0, "batch": 8, "heads": 40, "kv_heads": 40, "hd": 128,
         "nodes": 64, "context": 3000},
        # The smallest call: one short sequence with six rows (tiny block, 64-wide heads).  Latency alone.
        {"name": "attn_few_tiny", "kind": "attention", "kvq": 0, "batch": 1, "heads": 8, "kv_heads": 8, "hd": 64,
         "nodes": 6, "context": 51},
        # Trees of 26 rows checked, 7B-shaped block with a key head a query head, contexts to 612: the cache's bytes.
        {"name": "attn_bf16_7b", "kind": "attention", "kvq": 0, "batch": 8, "heads": 32, "kv_heads": 32, "hd": 128,
         "nodes": 26, "context": 612},
        # Trees of 16 rows checked, 70B-shaped block, int8 cache, 32 contexts to 2148: the cache's bytes, widened.
        {"name": "attn_int8_70b", "kind": "attention", "kvq": 1, "batch": 32, "heads": 64, "kv_heads": 8, "hd": 128,
         "nodes": 16, "context": 2148},
        # Large trees over long contexts, 70B-shaped block: products.
        {"name": "attn_bf16_70b_long", "kind": "attention", "kvq": 0, "batch": 8, "heads": 64, "kv_heads": 8, "hd": 128,
         "nodes": 64, "context": 8000},
        # The accepted path of 32 sequences with trees of up to 16 rows.
        {"name": "verify_32x16", "kind": "verify", "batch": 32, "nodes": 16, "vocab": 32000},
        # One sequence with a large tree over a large odd vocabulary: the latency of the way down.
        {"name": "verify_1x60", "kind": "verify", "batch": 1, "nodes": 60, "vocab": 100003},
        # Four beams each of 32 requests.
        {"name": "select_32x4", "kind": "select", "batch": 32, "beams": 4, "vocab": 32000},
        # One request with eight beams over a large odd vocabulary: few rows, long ones, most of them unaligned.
        {"name": "select_1x8", "kind": "select", "batch": 1, "beams": 8, "vocab": 128001},
        # The states of four beams each of 32 requests, 70B-shaped block, int8 cache.
        {"name": "reorder_int8_70b", "kind": "reorder", "kvq": 1, "batch": 32, "beams": 4, "kv_heads": 8, "hd": 128,
         "context": 2148},
        # Ten beams each of four requests, 13B-shaped block, bf16 cache.
        {"name": "reorder_bf16_13b", "kind": "reorder", "kvq": 0, "batch": 4, "beams": 10, "kv_heads": 40, "hd": 128,
         "context": 1000},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["cache", "attention", "attention", "attention", "verify", "select", "reorder"])
    if kind == "verify":
        batch, nodes = _log(rng, 1, 64), _log(rng, 1, 100)
        return {"kind": kind, "batch": batch, "nodes": nodes,
                "vocab": _log(rng, 1000, max(1001, min(200000, 16000000 // (batch * nodes))))}
    if kind == "select":
        batch, beams = _log(rng, 1, 64), _log(rng, 1, 16)
        return {"kind": kind, "batch": batch, "beams": beams,
                "vocab": _log(rng, 1000, max(1001, min(200000, 16000000 // (batch * beams))))}
    hd = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 8, 32])
    c = {"kind": kind, "kvq": rng.randint(0, 1), "batch": _log(rng, 1, 48)}
    if kind == "reorder":
        c.update(beams=_log(rng, 1, 16), kv_heads=kv_heads, hd=hd)
        # pages of all beams: at most 1 GB of them in bf16
        c["context"] = _log(rng, 4, max(5, min(8000, (1 << 30) // (c["batch"] * c["beams"] * kv_heads * hd * 4))))
        c["context"] += c["context"] % PAGE == 0  # a page part-filled, in one group at least
        return c
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 5, 7, 8, 16]) if kv_heads < 32 else 32
    c.update(heads=heads, kv_heads=kv_heads, hd=hd)
    if kind == "cache":
        c["nodes"] = _log(rng, 1, max(1, min(256, 512 * 120 // (c["batch"] * (heads + 2 * kv_heads)))))
        c["context"] = c["nodes"] + _log(rng, 1, 4000)
        return c
    c["nodes"] = _log(rng, 1, 256)
    # scores of the padded batch: at most those of the largest listed case
    limit = 8 * 64 * 64 * 8000
    if limit // (c["batch"] * heads * c["nodes"]) < 300:
        c["batch"] = max(1, limit // (300 * heads * c["nodes"]))
    most = limit // (c["batch"] * heads * c["nodes"])
    # and cached keys: at most those of the largest listed case
    most = min(most, 8 * 8 * 128 * 8000 // (c["batch"] * kv_heads * hd), 40000)
    c["context"] = _log(rng, max(1, min(32, most)), max(1, most))
    c["nodes"] = min(c["nodes"], c["context"])
    return c


def _lengths(case):
    """(rows, position of the first one) of each sequence: by the case alone."""
    r = random.Random("%(batch)d %(nodes)d" % case)
    B, most, T = case["batch"], case["nodes"], case.get("context", case["nodes"])
    n, pos = [], []
    for b in range(B):
        k = most if b == 0 else r.randint((most + 1) // 2, most)
        end = T if b == 0 else r.randint(max(k, T // 2), T)
        n.append(k)
        pos.append(end - k)
    return n, pos


def _starts(n):
    cu = [0]
    for k in n:
        cu.append(cu[-1] + k)
    return cu


def _beam_lengths(case):
    """Cached positions of each group of beams: by the case alone."""
    r = random.Random("%(batch)d %(beams)d %(context)d" % case)
    T = case["context"]
    return [T if b == 0 else r.randint(max(1, T // 2), T) for b in range(case["batch"])]


def _pools(case, g, pages, filled):
    """K and V pools and, for int8 codes, their scales; with values, or empty."""
    shape = (pages, case["kv_heads"], PAGE, case["hd"])
    c = {"pages": pages}
    for w in "kv":
        if case["kvq"] == 0:
            c[w] = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) if filled else torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
            continue
        if not filled:
            c[w], c[w + "s"] = torch.zeros(shape, dtype=torch.int8, device="cuda"), torch.zeros(shape[:3], device="cuda")
            continue
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16).float()
        c[w + "s"] = x.abs().amax(-1) / 127
        c[w] = (x / c[w + "s"][..., None]).round().clamp(-127, 127).to(torch.int8)
    return c


def _trees(n, seed):
    """Parents of every sequence's rows (row 0: -1), as a drafter grows them: a row hangs on any earlier one."""
    r = random.Random(seed)
    return [[-1] + [r.randint(0, i - 1) for i in range(1, k)] for k in n]


def _mask_words(trees, words):
    """The rows each row sees, itself and its ancestors, 32 to a word."""
    rows = []
    for t in trees:
        seen = []
        for i, p in enumerate(t):
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        rows += [[(s >> 32 * w) & 0xFFFFFFFF for w in range(words)] for s in seen]
    x = torch.tensor(rows, dtype=torch.int64, device="cuda")
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)


def _view(s):
    import paper_2501_13111_gb300 as fp

    c, case = s["cache"], s["case"]
    p = lambda w: c[w].data_ptr() if w in c else None  # noqa: E731
    return fp.fp_kv_view(case["kvq"], case["kv_heads"], case["hd"], PAGE, c["pps"], c["pages"], p("k"), p("v"), p("ks"),
                         p("vs"), p("table"))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    zeros = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": case, "err": zeros(1)}
    kind = case["kind"]
    if kind in ("cache", "attention"):
        n, pos = _lengths(case)
        cu = _starts(n)
        N, B, H, Hkv, hd = cu[-1], case["batch"], case["heads"], case["kv_heads"], case["hd"]
        trees = _trees(n, seed)
        # the cache: a shuffled page table that covers every sequence
        pps = max((p + k + PAGE - 1) // PAGE for p, k in zip(pos, n)) + 1
        pages = B * pps + 3
        s["cache"] = _pools(case, g, pages, kind == "attention")
        s["cache"].update(pps=pps, table=torch.randperm(pages, generator=g, device="cuda")[: B * pps].reshape(B, pps).to(torch.int32))
        s.update(N=N, B=B, H=H, Hkv=Hkv, hd=hd, max_new=max(n), max_len=max(p + k for p, k in zip(pos, n)))
        s.update(cu=i32(cu), pos=i32(pos), words=(max(n) + 31) // 32, row=(H + 2 * Hkv) * hd)
        # the rows' fused QKV, as the projection writes them
        x = torch.randn((N, s["row"]), generator=g, device="cuda")
        if kind == "attention":
            s["qkv"] = (1.5 * x).to(torch.bfloat16)
            s["mask"] = _mask_words(trees, s["words"])
            s["out"] = torch.zeros((N, H * hd), dtype=torch.bfloat16, device="cuda")
        else:
            s["qkv"] = x.to(torch.bfloat16)
            s["parent"] = i32([p for t in trees for p in t])
            # an accepted path: some row's way down from the root
            r = random.Random(seed + 1)
            path = []
            for t in trees:
                way, i = [], r.randrange(len(t))
                while i >= 0:
                    way.insert(0, i)
                    i = t[i]
                path += way + [-1] * (len(t) - len(way))
            s["path"] = i32(path)
            i = torch.arange(hd // 2, dtype=torch.float64, device="cuda")
            a = torch.arange(pps * PAGE, dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (-2 * i / hd)
            s["cs"] = torch.stack([a.cos(), a.sin()], -1).float().contiguous()
            s.update(depth=zeros(N), mask=zeros(N, s["words"]))
            for w, h in (("q", H), ("k", Hkv), ("v", Hkv)):
                s[w] = torch.zeros((N, h * hd), dtype=torch.bfloat16, device="cuda")
        if own:
            import paper_2501_13111_gb300 as fp

            s["view"] = _view(s)
            if kind == "attention":
                s["ws_bytes"] = fp.fp_op_attention_tree_workspace_bytes(B, H, Hkv, hd, s["max_new"])
                s["ws"] = torch.zeros(s["ws_bytes"], dtype=torch.uint8, device="cuda")
        return s
    if kind == "reorder":
        B, W, Hkv, hd = case["batch"], case["beams"], case["kv_heads"], case["hd"]
        n = _beam_lengths(case)
        pps = (max(n) + PAGE - 1) // PAGE + 1
        pages = B * W * pps
        s["cache"] = _pools(case, g, pages, True)
        own_pages = torch.randperm(pages, generator=g, device="cuda").reshape(B, W, pps)
        # full pages are shared by beams with the same history; part-filled and unused ones are each beam's own
        full = (i32(n) // PAGE)[:, None, None] > torch.arange(pps, device="cuda")
        came = torch.randint(0, W, (B, W, pps), generator=g, device="cuda")
        table = torch.where(full, own_pages.gather(1, came), own_pages).to(torch.int32).reshape(B * W, pps)
        s["cache"].update(pps=pps, table=torch.zeros_like(table))  # what the cache's view reads: the reordered one
        s.update(B=B, W=W, Hkv=Hkv, hd=hd, table=table, lens=i32(n))
        s["parent"] = torch.randint(0, W, (B, W), generator=g, device="cuda").sort(-1).values.to(torch.int32).reshape(-1)
        s.update(src=zeros(B * W), dst=zeros(B * W), rows=zeros(B * W))
        # what is looked at: every beam's rows of the part-filled page
        rem = [k % PAGE for k in n for _ in range(W)]
        s.update(N=sum(rem), cu=i32(_starts(rem)), pos=i32([k - k % PAGE for k in n for _ in range(W)]))
        for w in "kv":
            s[w] = torch.zeros((s["N"], Hkv * hd), dtype=torch.bfloat16, device="cuda")
        if own:
            s["view"] = _view(s)
        return s
    V = case["vocab"]
    if kind == "select":
        B, W = case["batch"], case["beams"]
        s.update(B=B, W=W, V=V, end=2)
        s["logits"] = 3 * torch.randn((B * W, V), generator=g, device="cuda")
        s["logits"][:, 7::97] = -math.inf  # tokens that a request has banned
        s["score"] = (-4 - 6 * torch.rand((B, W), generator=g, device="cuda")).sort(-1, descending=True).values.reshape(-1)
        s["done"] = (torch.rand(B * W, generator=g, device="cuda") < 0.1).to(torch.int32)  # some have met their end
        s.update(parent=zeros(B * W), token=zeros(B * W), new_done=zeros(B * W), new_score=torch.zeros(B * W, device="cuda"))
        if own:
            import paper_2501_13111_gb300 as fp

            s["ws_bytes"] = fp.fp_op_beam_select_workspace_bytes(B, W, V)
            s["ws"] = torch.zeros(s["ws_bytes"], dtype=torch.uint8, device="cuda")
        return s
    # verify: distributions with a few likely tokens, drafted from those
    n, _ = _lengths(case)
    cu = _starts(n)
    N, B = cu[-1], case["batch"]
    trees = _trees(n, seed)
    logits = 2 * torch.randn((N, V), generator=g, device="cuda")
    likely = torch.randint(0, V // 8, (N, 8), generator=g, device="cuda") * 8 + torch.arange(8, device="cuda")
    logits.scatter_(1, likely, math.log(V) + 2 + (2 - torch.arange(8, device="cuda")).expand(N, 8))
    s["p"] = torch.softmax(logits, -1)
    at, born = [], []  # of every row: its parent's row, and which child of it it is
    for c, t in zip(cu, trees):
        count = [0] * len(t)
        for p in t:
            at.append(c + max(p, 0))
            born.append(count[p] if p >= 0 else 0)
            if p >= 0:
                count[p] += 1
    at, born = torch.tensor(at, device="cuda"), torch.tensor(born, device="cuda")
    s["tokens"] = torch.where(born < 8, likely[at, born % 8], (likely[at, 0] + born) % V).to(torch.int32)
    s["parent"] = i32([p for t in trees for p in t])
    s["u"] = torch.rand(N, generator=g, device="cuda")
    s.update(N=N, B=B, V=V, cu=i32(cu), path=zeros(N), out=zeros(N), n_out=zeros(B))
    return s


# ------------------------------------------------------------------ plain forms
def _rows(s):
    """Sequence and place in it of every row."""
    cu = s["cu"].long()
    t = torch.arange(s["N"], device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, t - cu[b]


def _ancestors(s, b, i, most):
    """[sequence, row, row]: whether the second is the first or an ancestor of it."""
    up = torch.zeros((s["B"], most, most), device="cuda")
    p = s["parent"].long()
    up[b, i, torch.where(p < 0, i, p)] = 1.0
    up[b, i, i] = 1.0
    for _ in range(max(1, (most - 1).bit_length())):  # ways of up to 1, 2, 4, .. steps
        up = (torch.matmul(up, up) > 0).float()
    return up


def _half(x):
    d = x.shape[-1] // 2
    return x[..., :d], x[..., d:]


def _plain_cache(s):
    c, H, Hkv, hd, N = s["cache"], s["H"], s["Hkv"], s["hd"], s["N"]
    b, i = _rows(s)
    words = s["words"]
    seen = _ancestors(s, b, i, 32 * words)[b, i]  # [N, 32 words]
    depth = seen.sum(-1).long() - 1
    bits = (seen.long().view(N, words, 32) << torch.arange(32, device="cuda")).sum(-1)
    mask = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32)
    pos = s["pos"].long()[b]

    def place(at):
        return c["table"].long()[b, at // PAGE], at % PAGE

    page, slot = place(pos + i)
    # the path's rows: where they come from, where they go
    path = s["path"].long()
    on = path >= 0
    src, dst = place(pos + path.clamp(min=0)), (page[on], slot[on])
    src = src[0][on], src[1][on]
    x = s["qkv"].view(N, H + 2 * Hkv, hd)
    cs = s["cs"][pos + depth][:, None]
    lo, hi = _half(x[:, : H + Hkv].float())
    cos, sin = cs[..., 0], cs[..., 1]
    qk = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(torch.bfloat16)
    back = []
    for w, y in (("k", qk[:, H:]), ("v", x[:, H + Hkv :])):
        if s["case"]["kvq"] == 0:
            c[w][page, :, slot] = y
            c[w][dst[0], :, dst[1]] = c[w][src[0], :, src[1]]
            back.append(c[w][page, :, slot].reshape(N, Hkv * hd))
            continue
        y = y.float()
        sc = y.abs().amax(-1) / 127
        code = torch.where(sc[..., None] > 0, (y / sc[..., None]).round(), torch.zeros_like(y)).clamp(-127, 127)
        c[w][page, :, slot] = code.to(torch.int8)
        c[w + "s"][page, :, slot] = sc
        c[w][dst[0], :, dst[1]] = c[w][src[0], :, src[1]]
        c[w + "s"][dst[0], :, dst[1]] = c[w + "s"][src[0], :, src[1]]
        back.append((c[w][page, :, slot].float() * c[w + "s"][page, :, slot][..., None]).to(torch.bfloat16).reshape(N, Hkv * hd))
    return {"depth": depth.to(torch.int32), "mask": mask, "q": qk[:, :H].reshape(N, H * hd), "k": back[0], "v": back[1]}


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
    q = torch.zeros((B, n, H, hd), device="cuda")  # the ragged trees side by side
    q[b, i] = s["qkv"][:, : H * hd].float().view(-1, H, hd)
    q = q.view(B, n, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, hd)
    sc = torch.matmul(q, kf.permute(0, 2, 3, 1)).view(B, Hkv, G, n, T)
    sc *= hd ** -0.5
    # of each key: the tree's row it belongs to (below 0: the prefix)
    j = key[None] - s["pos"].long()[:, None]
    word = torch.zeros((B, n, s["words"]), dtype=torch.int64, device="cuda")
    word[b, i] = s["mask"].long()
    at = j.clamp(0, 32 * s["words"] - 1)[:, None].expand(B, n, T)
    seen = (word.gather(2, at // 32) >> (at % 32) & 1).bool() & (j < 32 * s["words"])[:, None] | (j < 0)[:, None]
    sc.masked_fill_(~seen[:, None, None], -math.inf)
    sc -= sc.amax(-1, keepdim=True).clamp(min=-1e30)  # (rows of the padding see nothing)
    sc.exp_()
    sc /= sc.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(sc.view(B, Hkv, G * n, T), vf.permute(0, 2, 1, 3)).view(B, Hkv, G, n, hd)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, H * hd)[b, i].to(torch.bfloat16)


def _plain_verify(s):
    p, B, N = s["p"], s["B"], s["N"]
    cu = s["cu"].long()
    b, i = _rows(s)
    most = s["case"]["nodes"]
    cum = p.double().cumsum(-1)
    drawn = (cum > s["u"].double()[:, None] * cum[:, -1:]).to(torch.uint8).argmax(-1)  # after every row, followed or not
    par, tok = s["parent"].long(), s["tokens"].long()
    # whether a row is the one its parent's draw leads to: its token, and no earlier child has it
    up = (cu[b] + par).clamp(min=0)
    hit = (par >= 0) & (drawn[up] == tok)
    rival = (up[:, None] == up[None]) & hit[:, None] & hit[None] & (i[None] < i[:, None])
    hit &= ~rival.any(-1)
    miss = torch.ones((B, most), device="cuda")
    miss[b, i] = (~(hit | (i == 0))).float()
    seen = _ancestors(s, b, i, most)[b, i]
    on = (seen * miss[b]).sum(-1) == 0  # every row on the way from the root
    path = torch.full((N,), -1, dtype=torch.int64, device="cuda")
    out = path.clone()
    at = cu[b] + seen.sum(-1).long() - 1  # the path's rows stand in the order of their depth
    path[at[on]] = i[on]
    out[at[on]] = drawn[on]
    count = torch.zeros((B,), dtype=torch.int64, device="cuda").scatter_add_(0, b, on.long())
    return {"path": path.to(torch.int32), "tokens": out.to(torch.int32), "count": count.to(torch.int32)}


def _plain_select(s):
    B, W, V = s["B"], s["W"], s["V"]
    x = s["logits"].double()
    e = x - x.amax(-1, keepdim=True)
    x = e - e.exp().sum(-1, keepdim=True).log()
    done = (s["done"] != 0)[:, None]
    end = torch.arange(V, device="cuda") == s["end"]
    x = torch.where(done, torch.where(end, 0.0, -math.inf), x) + s["score"].double()[:, None]
    val, at = torch.topk(x.view(B, W * V), W)
    at, order = at.sort(-1)  # ties: the lowest index first
    val = val.gather(-1, order)
    val, order = val.sort(dim=-1, descending=True, stable=True)
    at = at.gather(-1, order)
    parent, token = at // V, at % V
    ended = (s["done"].view(B, W).gather(1, parent) != 0) | (token == s["end"])
    return {"parent": parent.reshape(-1).to(torch.int32), "token": token.reshape(-1).to(torch.int32),
            "score": val.reshape(-1).float(), "done": ended.reshape(-1).to(torch.int32)}


def _plain_reorder(s):
    c, B, W, N = s["cache"], s["B"], s["W"], s["N"]
    parent, table = s["parent"].long().view(B, W), s["table"].long().view(B, W, -1)
    beam, block = torch.arange(W, device="cuda"), torch.arange(table.shape[-1], device="cuda")
    tail, rem = (s["lens"].long() // PAGE)[:, None], (s["lens"].long() % PAGE)[:, None]
    child = parent[:, None, :] == beam[None, :, None]  # [B, beam, its children]
    has, first = child.any(-1), child.to(torch.uint8).argmax(-1)
    keeps = first.gather(1, parent) == beam
    free = has.long().argsort(dim=-1, stable=True)  # beams without children, in order
    rank = (~keeps).long().cumsum(-1) - 1
    page_of = torch.where(keeps, parent, free.gather(1, rank.clamp(min=0)))
    last = table.gather(2, tail[:, :, None].expand(B, W, 1))[..., 0]
    new = torch.where(block < tail[:, :, None], table.gather(1, parent[..., None].expand_as(table)), table)
    at_tail = (block == tail[:, :, None]) & (rem[:, :, None] > 0)
    new = torch.where(at_tail, last.gather(1, page_of)[..., None], new)
    copy = ~keeps & (rem > 0)
    src = torch.where(copy, last.gather(1, parent), -1).reshape(-1)
    dst = torch.where(copy, last.gather(1, page_of), -1).reshape(-1)
    rows = torch.where(copy, rem, 0).reshape(-1)
    # row by row of the copied pages
    i = torch.arange(PAGE, device="cuda")
    what, slot = (i[None] < rows[:, None]).nonzero(as_tuple=True)
    b, i = _rows(s)
    page, at = new.view(B * W, -1)[b, s["pos"].long()[b] // PAGE], i
    back = []
    for w in "kv":
        for t in (w, w + "s")[: 1 + s["case"]["kvq"]]:
            c[t][dst[what], :, slot] = c[t][src[what], :, slot]
        y = c[w][page, :, at]
        if s["case"]["kvq"]:
            y = (y.float() * c[w + "s"][page, :, at][..., None]).to(torch.bfloat16)
        back.append(y.reshape(N, s["Hkv"] * s["hd"]))
    return {"table": new.view(B * W, -1).to(torch.int32), "from": src.to(torch.int32), "to": dst.to(torch.int32),
            "rows": rows.to(torch.int32), "k": back[0], "v": back[1]}


# ------------------------------------------------------------------ the framework's calls
def _own_cache(s):
    import paper_2501_13111_gb300 as fp

    st = torch.cuda.current_stream().cuda_stream
    N, B, H, err, cu, pos = s["N"], s["B"], s["H"], s["err"].data_ptr(), s["cu"].data_ptr(), s["pos"].data_ptr()
    fp.fp_op_tree_plan(s["parent"].data_ptr(), N, B, cu, s["max_new"], s["depth"].data_ptr(), s["mask"].data_ptr(),
                       s["words"], err, st)
    fp.fp_op_rope_kv_tree(s["qkv"].data_ptr(), s["row"], N, B, H, s["view"], cu, pos, s["depth"].data_ptr(),
                          s["cs"].data_ptr(), s["q"].data_ptr(), H * s["hd"], err, st)
    fp.fp_op_kv_commit(s["view"], N, B, cu, pos, s["path"].data_ptr(), err, st)
    fp.fp_op_kv_read(s["view"], N, B, cu, pos, s["k"].data_ptr(), s["v"].data_ptr(), s["Hkv"] * s["hd"], err, st)
    return {"depth": s["depth"], "mask": s["mask"], "q": s["q"], "k": s["k"], "v": s["v"]}


def _own_attention(s):
    import paper_2501_13111_gb300 as fp

    fp.fp_op_attention_tree(s["qkv"].data_ptr(), s["row"], s["N"], s["B"], s["H"], s["view"], s["cu"].data_ptr(),
                            s["pos"].data_ptr(), s["mask"].data_ptr(), s["words"], s["max_new"], s["max_len"],
                            s["out"].data_ptr(), s["ws"].data_ptr(), s["ws_bytes"], s["err"].data_ptr(),
                            torch.cuda.current_stream().cuda_stream)
    return s["out"]


def _own_verify(s):
    import paper_2501_13111_gb300 as fp

    fp.fp_op_verify_tree(s["p"].data_ptr(), s["V"], s["N"], s["B"], s["cu"].data_ptr(), s["parent"].data_ptr(),
                         s["tokens"].data_ptr(), s["u"].data_ptr(), s["path"].data_ptr(), s["out"].data_ptr(),
                         s["n_out"].data_ptr(), s["err"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return {"path": s["path"], "tokens": s["out"], "count": s["n_out"]}


def _own_select(s):
    import paper_2501_13111_gb300 as fp

    fp.fp_op_beam_select(s["logits"].data_ptr(), s["V"], s["B"], s["W"], s["score"].data_ptr(), s["done"].data_ptr(),
                         s["end"], s["parent"].data_ptr(), s["token"].data_ptr(), s["new_score"].data_ptr(),
                         s["new_done"].data_ptr(), s["ws"].data_ptr(), s["ws_bytes"], s["err"].data_ptr(),
                         torch.cuda.current_stream().cuda_stream)
    return {"parent": s["parent"], "token": s["token"], "score": s["new_score"], "done": s["new_done"]}


def _own_reorder(s):
    import paper_2501_13111_gb300 as fp

    st = torch.cuda.current_stream().cuda_stream
    B, W, c, err = s["B"], s["W"], s["cache"], s["err"].data_ptr()
    fp.fp_op_beam_reorder(B, W, c["pps"], PAGE, s["lens"].data_ptr(), s["parent"].data_ptr(), s["table"].data_ptr(),
                          c["table"].data_ptr(), s["src"].data_ptr(), s["dst"].data_ptr(), s["rows"].data_ptr(), err, st)
    fp.fp_op_kv_copy(s["view"], B * W, s["src"].data_ptr(), s["dst"].data_ptr(), s["rows"].data_ptr(), err, st)
    fp.fp_op_kv_read(s["view"], s["N"], B * W, s["cu"].data_ptr(), s["pos"].data_ptr(), s["k"].data_ptr(),
                     s["v"].data_ptr(), s["Hkv"] * s["hd"], err, st)
    return {"table": c["table"], "from": s["src"], "to": s["dst"], "rows": s["rows"], "k": s["k"], "v": s["v"]}


_PLAIN = {"cache": _plain_cache, "attention": _plain_attention, "verify": _plain_verify, "select": _plain_select,
          "reorder": _plain_reorder}
_OWN = {"cache": _own_cache, "attention": _own_attention, "verify": _own_verify, "select": _own_select,
        "reorder": _own_reorder}


def run(state):
    kind = state["case"]["kind"]
    return _OWN[kind](state) if own else _PLAIN[kind](state)


def work(case):
    kind = case["kind"]
    if kind == "select":
        rows = case["batch"] * case["beams"]
        return {"bytes": 4 * rows * case["vocab"], "flops": 3 * rows * case["vocab"]}
    if kind == "verify":  # a row of probabilities a sequence at least, and the trees
        return {"bytes": 4 * case["batch"] * (case["vocab"] + 4 * case["nodes"]), "flops": case["batch"] * case["vocab"]}
    cached = 2 * case["kv_heads"] * (case["hd"] + 4 if case["kvq"] else 2 * case["hd"])  # bytes of a position
    if kind == "reorder":
        n, W = _beam_lengths(case), case["beams"]
        # tables read and written; a third of the beams copy (as many as have no child), every beam's rows read back
        rows = sum(k % PAGE for k in n) * W
        return {"bytes": 8 * W * sum(k // PAGE + 1 for k in n) + rows * (2 * cached / 3 + cached + 4 * case["kv_heads"] * case["hd"]),
                "flops": 0}
    n, pos = _lengths(case)
    H, Hkv, hd, N = case["heads"], case["kv_heads"], case["hd"], sum(n)
    if kind == "cache":
        return {"bytes": N * (2 * (H + 2 * Hkv) * hd + 2 * H * hd + 2 * cached + 4 * Hkv * hd), "flops": 6 * N * (H + Hkv) * hd}
    pairs = sum(k * p + k for p, k in zip(pos, n))  # the prefix and the row itself, at least
    return {"bytes": N * 4 * H * hd + cached * sum(p + k for p, k in zip(pos, n)), "flops": 4 * pairs * H * hd}


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_parents(s, b):
    lo, hi = s["cu"][b].item(), s["cu"][b + 1].item()
    return lo, hi, s["parent"][lo:hi].tolist()


def _exact_cache(s):
    H, Hkv, hd, cu, pos = s["H"], s["Hkv"], s["hd"], s["cu"].tolist(), s["pos"].tolist()
    depth, words, order, at = [], [], [], []
    for b in range(s["B"]):
        lo, hi, par = _exact_parents(s, b)
        chains = []
        for i in range(hi - lo):
            chain, j = [i], par[i]
            while j >= 0:
                chain.append(j)
                j = par[j]
            chains.append(chain)
            depth.append(len(chain) - 1)
            at.append(pos[b] + len(chain) - 1)
            m = sum(1 << j for j in chain)
            words.append([int.from_bytes(((m >> 32 * w) & 0xFFFFFFFF).to_bytes(4, "little"), "little", signed=True) for w in range(s["words"])])
            w = s["path"][lo + i].item()
            order.append(lo + (w if w >= 0 else i))  # what the row's place holds in the end
    ang = torch.tensor(at).double()[:, None] * ROPE_BASE ** (-2 * torch.arange(hd // 2).double() / hd)
    turn = torch.polar(torch.ones_like(ang), ang).cuda()[:, None]
    x = s["qkv"].double().view(s["N"], -1, hd)
    z = torch.complex(x[:, : H + Hkv, : hd // 2], x[:, : H + Hkv, hd // 2 :]) * turn
    qk = torch.cat([z.real, z.imag], -1)
    res = {"depth": torch.tensor(depth, dtype=torch.int32), "mask": torch.tensor(words, dtype=torch.int32), "q": qk[:, :H].flatten(1)}
    for w, y in (("k", qk[:, H:]), ("v", x[:, H + Hkv :])):
        y = y[torch.tensor(order).cuda()]
        if s["case"]["kvq"]:
            y = y.to(torch.bfloat16).double()  # what is quantised
            m = y.abs().max(-1, keepdim=True).values.clamp(min=1e-300)
            y = torch.round(y / m * 127) * (m / 127)
        res[w] = y.flatten(1)
    return res


def _exact_attention(s):
    c, H, Hkv, hd = s["cache"], s["H"], s["Hkv"], s["hd"]
    cu, pos = s["cu"].tolist(), s["pos"].tolist()
    out = torch.zeros((s["N"], H, hd), dtype=torch.float64, device="cuda")
    x = s["qkv"][:, : H * hd].double().view(s["N"], H, hd)
    for b in range(s["B"]):
        lo, hi = cu[b], cu[b + 1]
        L = pos[b] + hi - lo
        kv = {}
        for w in "kv":
            y = c[w][c["table"][b].long()].double()  # pages, heads, slots, hd
            if s["case"]["kvq"]:
                y = y * c[w + "s"][c["table"][b].long()].double().unsqueeze(-1)
            kv[w] = y.transpose(0, 1).flatten(1, 2)[:, :L]
        seen = torch.ones((hi - lo, L), dtype=torch.bool)
        for i, row in enumerate(s["mask"][lo:hi].tolist()):
            m = sum((w & 0xFFFFFFFF) << 32 * k for k, w in enumerate(row))
            seen[i, pos[b] :] = torch.tensor([m >> j & 1 for j in range(hi - lo)], dtype=torch.bool)
        seen = seen.cuda()
        for h in range(H):
            z = x[lo:hi, h] @ kv["k"][h // (H // Hkv)].T / math.sqrt(hd)
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            out[lo:hi, h] = torch.softmax(z, -1) @ kv["v"][h // (H // Hkv)]
    return out.flatten(1)


def _exact_verify(s):
    path, out, count = [], [], []
    for b in range(s["B"]):
        lo, hi, par = _exact_parents(s, b)
        tok = s["tokens"][lo:hi].tolist()
        way, drawn, c = [], [], 0
        while c >= 0:
            total = s["p"][lo + c].double().cpu().cumsum(0)
            t = int(torch.searchsorted(total, s["u"][lo + c].double().cpu() * total[-1], right=True))
            way.append(c)
            drawn.append(t)
            c = next((j for j in range(c + 1, hi - lo) if par[j] == c and tok[j] == t), -1)
        count.append(len(way))
        path += way + [-1] * (hi - lo - len(way))
        out += drawn + [-1] * (hi - lo - len(way))
    return {"path": torch.tensor(path, dtype=torch.int32), "tokens": torch.tensor(out, dtype=torch.int32),
            "count": torch.tensor(count, dtype=torch.int32)}


def _exact_select(s):
    W, V = s["W"], s["V"]
    res = {"parent": [], "token": [], "score": [], "done": []}
    score, done = s["score"].double().tolist(), s["done"].tolist()
    for b in range(s["B"]):
        found = []
        for w in range(W):
            r = b * W + w
            if done[r]:
                found.append((-score[r], w, s["end"]))
                continue
            x = s["logits"][r].double()
            x = x - torch.logsumexp(x, 0) + score[r]
            order = torch.sort(x, descending=True, stable=True)
            found += [(-v, w, t) for v, t in zip(order.values[:W].tolist(), order.indices[:W].tolist())]
        for v, w, t in sorted(found)[:W]:
            res["parent"].append(w)
            res["token"].append(t)
            res["score"].append(-v)
            res["done"].append(int(bool(done[b * W + w]) or t == s["end"]))
    return {k: torch.tensor(v, dtype=torch.float64 if k == "score" else torch.int32) for k, v in res.items()}


def _exact_reorder(s):
    c, B, W, Hkv, hd = s["cache"], s["B"], s["W"], s["Hkv"], s["hd"]
    old, par, lens = s["table"].view(B, W, -1).tolist(), s["parent"].view(B, W).tolist(), s["lens"].tolist()
    table, move, looked = [], [], []
    for b in range(B):
        t, rem = divmod(lens[b], PAGE)
        spare = [w for w in range(W) if w not in par[b]]
        met = set()
        for w, p in enumerate(par[b]):
            row = old[b][p][:t] + old[b][w][t:]
            held = old[b][p][t]
            if rem and p in met:
                row[t] = old[b][spare.pop(0)][t]
                move.append((held, row[t], rem))
            else:
                row[t] = held if rem else row[t]
                move.append((-1, -1, 0))
            met.add(p)
            table.append(row)
            looked += [(held, i) for i in range(rem)]  # what the beam's rows have to be: its parent's
    page, slot = (torch.tensor([x[i] for x in looked], dtype=torch.int64, device="cuda") for i in (0, 1))
    res = {"table": torch.tensor(table, dtype=torch.int32)}
    res.update({k: torch.tensor([m[i] for m in move], dtype=torch.int32) for i, k in enumerate(("from", "to", "rows"))})
    for w in "kv":
        y = c[w][page, :, slot].double()
        if s["case"]["kvq"]:
            y = y * c[w + "s"][page, :, slot].double().unsqueeze(-1)
        res[w] = y.reshape(len(looked), Hkv * hd)
    return res


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"cache": _exact_cache, "attention": _exact_attention, "verify": _exact_verify, "select": _exact_select,
            "reorder": _exact_reorder}[case["kind"]](s)
