"""TEST INFRASTRUCTURE: the oracle of the calls around a paged cache, in plain fp64 numpy: head norms with the rotation by position,
rows into pages, attention over pages.  Written as the definitions of include/dd.h state them: one row, one page, one sequence at a
time.  Neither imports nor is imported by the HIP library's package.

Arrays hold numbers, not storage bits: a cache in e4m3 is the array of the values that its codes stand for, with its scales beside it.
"""
from __future__ import annotations

import numpy as np

E4M3_MAX = 448.0


def e4m3(x):
    """The e4m3 number nearest to x, ties to the even significand; |x| <= 448."""
    x = np.asarray(x, np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.rint(x / step) * step


def e4m3_step(x):
    """Distance of the e4m3 numbers around |x|."""
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(np.asarray(x, np.float64)), 2.0 ** -6))) - 3)


def norm_rope_row(x, weight, eps, inv_freq, position, interleaved):
    y = np.array(x, np.float64)
    d = len(y)
    if weight is not None:
        y = y / np.sqrt(np.sum(y * y) / d + eps) * np.asarray(weight, np.float64)
    half = 0 if inv_freq is None else len(inv_freq)
    out = y.copy()
    for k in range(half):
        i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + half)
        a = float(position) * float(inv_freq[k])
        out[i] = y[i] * np.cos(a) - y[j] * np.sin(a)
        out[j] = y[j] * np.cos(a) + y[i] * np.sin(a)
    return out


def norm_rope(x, weight, eps, inv_freq, positions, interleaved):
    """x [B, heads, n, d]; positions [B, n] -> [B, heads, n, d]"""
    out = np.empty(np.shape(x), np.float64)
    for b, h, i in np.ndindex(*out.shape[:3]):
        out[b, h, i] = norm_rope_row(x[b, h, i], weight, eps, inv_freq, positions[b][i], interleaved)
    return out


def scale_for(a):
    """2^e with the least e >= -126 such that a <= 448 * 2^e"""
    e = -126
    while a > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def paged_append(Kc, Vc, k_scale, v_scale, K, V, table, starts, kv_lens=None, n_rows=None, weight=None, eps=1e-6, inv_freq=None,
                 interleaved=False):
    """Kc [pages, Hkv, P, d], Vc [pages, Hkv, d, P]; scales [pages, Hkv] or None (pages without codes: rows are kept as they are, the
    rounding of storage is the caller's); K, V [B, Hkv, n, d].  Returns new (Kc, Vc, k_scale, v_scale) and `raw`, the same caches
    with what the rows were before their rounding, in units of their scale."""
    Kn, Vn = np.array(Kc, np.float64), np.array(Vc, np.float64).swapaxes(-1, -2).copy()
    fp8 = k_scale is not None
    ks, vs = (np.array(k_scale, np.float64), np.array(v_scale, np.float64)) if fp8 else (None, None)
    Kraw, Vraw = Kn.copy(), Vn.copy()
    pages, Hkv, P, _ = Kn.shape
    B, _, n, _ = np.shape(K)
    for b in range(B):
        start = int(starts[b])
        count = n if n_rows is None else min(max(int(n_rows[b]), 0), n)
        held = start if kv_lens is None else int(kv_lens[b])
        at = {}                                               # page of the table -> positions written there
        for r in range(count):
            p = start + r
            if 0 <= p < len(table[b]) * P:
                at.setdefault(p // P, []).append(p)
        for j, positions in at.items():
            page = int(table[b][j])
            if not 0 <= page < pages:
                continue
            kept = [p for p in range(j * P, min((j + 1) * P, max(held, 0))) if p not in positions]
            for g in range(Hkv):
                for cache, raw, scale, rows in ((Kn, Kraw, ks, "k"), (Vn, Vraw, vs, "v")):
                    if rows == "k":
                        new = {p: norm_rope_row(K[b, g, p - start], weight, eps, inv_freq, p, interleaved) for p in positions}
                    else:
                        new = {p: np.asarray(V[b, g, p - start], np.float64) for p in positions}
                    s = 1.0
                    if fp8:
                        s = scale_for(max(np.abs(x).max() for x in new.values()))
                        if kept:
                            s = max(s, scale[page, g])
                            for p in kept:
                                raw[page, g, p % P] = cache[page, g, p % P] * scale[page, g] / s
                                cache[page, g, p % P] = e4m3(raw[page, g, p % P])
                        scale[page, g] = s
                    for p, x in new.items():
                        raw[page, g, p % P] = x / s
                        cache[page, g, p % P] = e4m3(x / s) if fp8 else x
    return Kn, Vn.swapaxes(-1, -2), ks, vs, (Kraw, Vraw.swapaxes(-1, -2))


def paged_attention(Q, Kc, Vc, k_scale, v_scale, table, kv_lens):
    """Q [B, H, n, d] -> (O, A): the attention, and the same weights over the values' magnitudes (what its rounding is relative to)."""
    B, H, n, d = np.shape(Q)
    pages, Hkv, P, _ = np.shape(Kc)
    O, A = np.zeros((B, H, n, d)), np.zeros((B, H, n, d))
    for b in range(B):
        held = min(max(int(kv_lens[b]), 0), len(table[b]) * P)
        keys = [(int(table[b][p // P]), p % P) for p in range(held)]
        keys = [(page, slot) for page, slot in keys if 0 <= page < pages]
        if not keys:
            continue
        page, slot = np.array([k[0] for k in keys]), np.array([k[1] for k in keys])
        for h in range(H):
            g = h * Hkv // H
            k = np.asarray(Kc, np.float64)[page, g, slot]
            v = np.asarray(Vc, np.float64)[page, g, :, slot]
            if k_scale is not None:
                k = k * np.asarray(k_scale, np.float64)[page, g][:, None]
                v = v * np.asarray(v_scale, np.float64)[page, g][:, None]
            s = np.asarray(Q[b, h], np.float64) @ k.T / np.sqrt(d)
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            O[b, h], A[b, h] = w @ v, w @ np.abs(v)
    return O, A
