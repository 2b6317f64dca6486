"""Chunks of new tokens: probabilities and the verification of drafted tokens, in fp64.

Attention of a chunk is ``model.attention`` with the chunk's positions; the append is ``model.rope`` and the cache's
quantiser.  The verification follows speculative sampling as its authors define it (Leviathan, Kalman and Matias, ICML
2023; Chen et al., arXiv 2302.01318): a draft t ~ q is kept with probability min(1, p(t)/q(t)), else a token is drawn
from the normalised positive part of p - q, so that what comes out is distributed as p.
"""
from __future__ import annotations

import numpy as np


def probabilities(logits, temperature=None):
    """softmax(logits / T) of each row; T = 0: 1 at the first maximum; a row of -inf: zeros."""
    x = np.asarray(logits, np.float64)
    out = np.zeros_like(x)
    t = np.ones(len(x)) if temperature is None else np.asarray(temperature, np.float64)
    for m, row in enumerate(x):
        if not (t[m] >= 0) or np.isinf(t[m]) or np.all(row == -np.inf):
            continue
        if t[m] == 0:
            out[m, int(np.argmax(row))] = 1.0
            continue
        with np.errstate(invalid="ignore"):
            e = np.exp((row - np.max(row)) / t[m])
            out[m] = e / np.sum(e)
    return out


def draw(w, r):
    """The lowest token whose running sum exceeds r times the whole; past the end the last that has a weight."""
    w = np.where(w > 0, w, 0.0)
    c = np.cumsum(w)
    at = np.nonzero(c > r * c[-1])[0]
    return int(at[0]) if len(at) else int(np.nonzero(w)[0][-1])


def verify(p, q, tokens, u, r):
    """One sequence: p [k+1][V], q [k+1][V] or None, tokens [k+1] (the first is not read), u [k+1], r.
    Returns (emitted tokens, all good): the accepted drafts and the drawn token, if one could be drawn."""
    p = np.asarray(p, np.float64)
    k, V = len(p) - 1, p.shape[1]
    out, ok = [], True
    a = 0
    while a < k:
        t = int(tokens[a + 1])
        if not 0 <= t < V:
            ok = False
            break
        qt = 1.0 if q is None else float(q[a][t])
        if not float(u[a]) * qt < p[a][t]:
            break
        out.append(t)
        a += 1
    w = p[a]
    if a < k:
        rest = p[a].copy()
        if q is None:
            if 0 <= int(tokens[a + 1]) < V:
                rest[int(tokens[a + 1])] = 0.0
        else:
            rest = np.asarray(p[a], np.float64) - np.asarray(q[a], np.float64)
        rest = np.where(rest > 0, rest, 0.0)
        w = rest if np.sum(rest) > 0 else w
    w = np.where(w > 0, w, 0.0)
    s = np.sum(w)
    if not (s > 0 and np.isfinite(s)):
        return out, False
    return out + [draw(w, float(r))], ok
