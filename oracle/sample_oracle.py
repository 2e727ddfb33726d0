"""Plain fp64 CPU oracle of sampling with temperature, top-k, top-p and min-p.

TEST INFRASTRUCTURE.  Only ``tests/`` may import, call or time this module.  It
shares no code with the HIP path.

Per row: the candidates are ranked by logit (descending), then token (ascending);
top-k keeps a prefix of the ranking, top-p the shortest prefix of that whose mass
reaches p of its mass, min-p what weighs at least min_p of the best; the token is
the first in vocabulary order whose running sum of kept weights exceeds u times
their total.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["kept_tokens", "sample_row", "sample"]


def kept_tokens(z, allowed=None, T=1.0, k=0, p=1.0, min_p=0.0):
    """(tokens in rank order, their weights) that the rules keep of one row."""
    z = np.asarray(z, dtype=np.float64)
    ok = ~np.isnan(z) & (z > -np.inf)
    if allowed is not None:
        ok &= np.asarray(allowed, dtype=bool)
    cand = np.flatnonzero(ok)
    rank = cand[np.argsort(-z[cand], kind="stable")]
    if rank.size == 0:
        return rank, np.zeros(0)
    if not T > 0:
        return rank[:1], np.ones(1)
    best = z[rank[0]]
    w = np.array([1.0 if z[v] == best else math.exp((z[v] - best) / T) for v in rank])
    if k > 0:
        rank, w = rank[:k], w[:k]
    if not p >= 1:
        target = (p if p > 0 else 0.0) * math.fsum(w)
        n, mass = 0, 0.0
        while n < len(w) and (n == 0 or mass < target):
            mass += w[n]
            n += 1
        rank, w = rank[:n], w[:n]
    if min_p > 0:
        keep = w >= min(min_p, 1.0)
        rank, w = rank[keep], w[keep]
    return rank, w


def sample_row(z, u, **rules):
    """The token of one row, -1 without candidates."""
    rank, w = kept_tokens(z, **rules)
    if rank.size == 0:
        return -1
    order = np.argsort(rank)
    rank, w = rank[order], w[order]
    u = 0.0 if not u > 0 else min(float(u), 1.0 - 2.0 ** -24)
    upto = np.cumsum(w)
    hit = np.flatnonzero(upto > u * upto[-1])
    return int(rank[hit[0]] if hit.size else rank[np.flatnonzero(w > 0)[-1]])


def sample(logits, u, M, mask=None, T=None, k=None, p=None, min_p=None, prev=None):
    """(tokens, scores) of all rows; rules are arrays over requests or None, mask bool [R, V]."""
    z = np.asarray(logits, dtype=np.float64)
    R, V = z.shape
    tokens, scores = np.empty(R, dtype=np.int32), np.empty(R)
    for r in range(R):
        b = r // M
        rules = dict(allowed=None if mask is None else mask[r], T=1.0 if T is None else float(T[b]),
                     k=0 if k is None else int(k[b]), p=1.0 if p is None else float(p[b]),
                     min_p=0.0 if min_p is None else float(min_p[b]))
        t = tokens[r] = sample_row(z[r], u[r], **rules)
        if t < 0:
            scores[r] = -np.inf
            continue
        with np.errstate(invalid="ignore"):
            top = z[r].max()
            logp = z[r, t] - top - np.log(np.exp(z[r] - top).sum())
        scores[r] = (0.0 if prev is None else float(prev[r])) + logp
    return tokens, scores
