"""Several continuations of a sequence: trees of drafted tokens, and beams, in fp64 and plain loops.

Attention of a tree is ``attention`` below with each row's own set of keys; the append is ``model.rope`` at the prefix'
length plus the row's depth, and the cache's quantiser.  A tree is verified by drawing from the target itself: a draft
is accepted when it is what was drawn, so the tokens are distributed as the target says, whatever the drafts are.
"""
from __future__ import annotations

import numpy as np

from oracle import chunk

LEAST = 2.0 ** 128 - 2.0 ** 103  # from here on down a score rounds to fp32's -inf


def plan(parent):
    """Depth of each row and the set of rows it sees (itself and its ancestors); an impossible parent: none."""
    depth, seen, good = [], [], True
    for i, p in enumerate(parent):
        if not -1 <= p < i:
            p, good = -1, False
        depth.append(0 if p < 0 else depth[p] + 1)
        seen.append({i} | (set() if p < 0 else seen[p]))
    return depth, seen, good


def words(seen, stride):
    """Sets of rows as uint32 mask words [rows][stride]."""
    out = np.zeros((len(seen), stride), np.uint32)
    for i, s in enumerate(seen):
        for j in s:
            if j // 32 < stride:
                out[i, j // 32] |= np.uint32(1 << (j % 32))
    return out


def attention(q, visible, k, v):
    """q [n][H][hd]; visible bool [n][L]; k, v [L][Hkv][hd] -> [n][H][hd]; a row that sees nothing: zeros."""
    n, H, hd = q.shape
    group = H // k.shape[1]
    out = np.zeros((n, H, hd))
    for h in range(H):
        s = q[:, h] @ k[:, h // group].T / np.sqrt(hd)
        s = np.where(visible, s, -np.inf)
        m = np.max(s, -1, keepdims=True, initial=-np.inf)
        e = np.where(visible, np.exp(s - np.where(np.isfinite(m), m, 0.0)), 0.0)
        z = e.sum(-1, keepdims=True)
        out[:, h] = (e / np.where(z > 0, z, 1.0)) @ v[:, h // group]
    return out


def verify(p, parent, tokens, u):
    """One tree: p [n][V], u [n].  Returns (path, drawn tokens, all good)."""
    path, out, c = [], [], 0
    while True:
        path.append(c)
        w = np.asarray(p[c], np.float64)
        w = np.where(w > 0, w, 0.0)
        s = np.sum(w)
        if not (s > 0 and np.isfinite(s)):
            return path, out, False
        t = chunk.draw(w, float(u[c]))
        out.append(t)
        nxt = [i for i in range(c + 1, len(parent)) if parent[i] == c and tokens[i] == t]
        if not nxt:
            return path, out, True
        c = nxt[0]


def select(logits, score, done, end):
    """One group: logits [W][V], score [W], done [W].  Returns ([(parent, token, score, done)] * W, all good)."""
    W, V = logits.shape
    found, good = [], True
    for w in range(W):
        s = float(score[w])
        if s == -np.inf:
            continue
        if not np.isfinite(s):
            good = False
            continue
        if done[w]:
            found.append((-s, w, 0, end))
            continue
        x = np.asarray(logits[w], np.float64)
        if np.any(np.isnan(x)) or np.any(x == np.inf):
            good = False
            continue
        m = np.max(x)
        if m == -np.inf:
            continue
        z = np.log(np.sum(np.exp(x - m)))  # (against m: x - lse would lose z where m is far from zero)
        order = np.lexsort((np.arange(V), -x))[:W]
        for i, t in enumerate(order):
            v = s + ((x[t] - m) - z)
            if x[t] > -np.inf and v > -LEAST:
                found.append((-v, w, i, int(t)))  # (a beam's order is its logits', where v does not tell them apart)
    found.sort()
    out = [(w, t, -v, int(bool(done[w]) or t == end)) for v, w, _, t in found[:W]]
    return out + [(-1, -1, -np.inf, 0)] * (W - len(out)), good


def reorder(table, length, parent, page=16):
    """One group: table [W][pps], its cached positions, parent [W].  Returns (new table, copies (from, to, rows) or
    (-1, -1, 0) of each beam, all good)."""
    table = np.asarray(table)
    W, pps = table.shape
    none = (-1, -1, 0)
    if not 0 <= length <= pps * page:
        return table.copy(), [none] * W, False
    good = all(-1 <= p < W for p in parent)
    parent = [p if -1 <= p < W else -1 for p in parent]
    full, rem = divmod(length, page)
    new, copies = table.copy(), [none] * W
    free = [x for x in range(W) if x not in parent]
    met = set()
    for w, p in enumerate(parent):
        if p >= 0:
            new[w, :full] = table[p, :full]
        holder = p
        if p < 0 or p in met:
            holder = free.pop(0)
        if rem:
            new[w, full] = table[holder, full]
            if p >= 0 and p in met:
                copies[w] = (int(table[p, full]), int(table[holder, full]), rem)
        met.add(p)
    return new, copies, good
