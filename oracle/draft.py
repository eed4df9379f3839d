"""TEST INFRASTRUCTURE: the oracle of the verification of drafted tokens, in plain fp64 numpy, as include/dd.h states it: one sequence,
one draft, one token at a time.  Neither imports nor is imported by the HIP library's package."""
from __future__ import annotations

import numpy as np


def probabilities(logits, temperature):
    x = np.asarray(logits, np.float64)
    if not temperature > 1e-6:
        p = np.zeros_like(x)
        p[int(np.argmax(x))] = 1.0                            # (the first of the largest)
        return p
    e = np.exp((x - x.max()) / float(temperature))
    return e / e.sum()


def draw(weights, u):
    """(the lowest x whose running sum is more than u times the whole, the distance of that mark to the nearest border relative to the
    whole)"""
    c = np.cumsum(weights)
    mark = u * c[-1]
    x = int(np.searchsorted(c, mark, side="right"))
    near = np.abs(c[max(0, x - 1):x + 1] - mark).min()
    return min(x, int(np.flatnonzero(weights)[-1])), near / c[-1]


def verify_draft(logits_v, logits_d, tokens, uniforms, temperature=None, n_draft=None, bonus=True):
    """-> (tokens [B,n+1], accepted [B], chances [B,n], margin [B]): how far, relative to the probabilities compared, the closest decision
    of a sequence was from going the other way."""
    B, n = np.shape(tokens)
    V = np.shape(logits_v)[-1]
    out, accepted, chances = np.full((B, n + 1), -1, np.int32), np.zeros(B, np.int32), np.zeros((B, n))
    margin = np.full(B, np.inf)
    for b in range(B):
        t = 1.0 if temperature is None else float(temperature[b])
        drafts = n if n_draft is None else min(max(int(n_draft[b]), 0), n)
        weights = None
        for i in range(drafts):
            x = int(tokens[b][i])
            p = probabilities(logits_v[b][i], t)
            if logits_d is None:
                q = np.zeros(V)
                if 0 <= x < V:
                    q[x] = 1.0
                qx = 1.0
            else:
                q = probabilities(logits_d[b][i], t)
                qx = q[x] if 0 <= x < V else 0.0
            px = p[x] if 0 <= x < V else 0.0
            chances[b, i] = px / qx if qx > px else float(px > 0)
            if weights is not None:
                continue
            u = float(uniforms[b][i])
            if t > 1e-6 and max(px, u * qx) > 0:
                margin[b] = min(margin[b], abs(u * qx - px) / max(px, u * qx))
            if u * qx < px:
                out[b, i] = x
                accepted[b] += 1
            else:
                weights = np.maximum(p - q, 0.0)
                if not weights.sum() > 0:
                    weights = p
        a = accepted[b]
        if weights is None and bonus:
            weights = probabilities(logits_v[b][a], t)
        if weights is not None:
            out[b, a], near = draw(weights, max(float(uniforms[b][n]), 0.0))
            if t > 1e-6:
                margin[b] = min(margin[b], near * weights.sum())
    return out, accepted, chances, margin
