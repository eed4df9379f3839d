"""How exact the rotation is where that shows: fp32 rows to their last bits, keys on e4m3 pages next to a border between two codes."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from _paged import dev, host, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("far", [200, 200000, 2**31 - 1])
def test_fp32_rotation(far, interleaved):
    # In units of 2^-24, for a pair of length r.  The angle from the nearest quarter of a turn, at most pi / 4, is rounded once: 0.5.  The sine:
    # x^3 P is at most 0.081 and carries three roundings, 0.25, the last sum 0.5, what the series leaves out 0.03; the cosine: x^2 R is at
    # most 0.29 and carries one, R's own is 0.25 times x^2 = 0.62, with later terms 0.5 in all, the last difference 0.5: 1 each, sqrt 2 r
    # together.  Two products of lengths that add to r at most, 1 r; their sum, 1 r: under 4 r.
    import torch
    rng = np.random.default_rng(far % 1000 + interleaved)
    d, n = 128, 4096
    x = rng.standard_normal((1, 2, n, d)).astype(np.float32)
    f = (500000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    pos = rng.integers(-far, far, (1, n))
    got, _ = dd.dd_qk_norm_rope(dev(x), inv_freq=dev(f), positions=ints(pos), interleaved=interleaved)
    a = pos[0].astype(np.longdouble)[:, None] * f.astype(np.longdouble)
    c, s = np.cos(a).astype(np.float64), np.sin(a).astype(np.float64)
    pair = (lambda y: (y[..., 0::2], y[..., 1::2])) if interleaved else (lambda y: (y[..., :d // 2], y[..., d // 2:]))
    (u, v), (gu, gv) = pair(x.astype(np.float64)), pair(host(got))
    r = np.hypot(u, v)
    worst = max((np.abs(gu - (u * c - v * s)) / r).max(), (np.abs(gv - (v * c + u * s)) / r).max())
    assert worst <= 4.25 * 2.0 ** -24, f"{worst * 2.0 ** 24:.2f} x 2^-24"


@pytest.mark.parametrize("seed", [1, 2])
def test_codes_of_rotated_keys(seed):
    # A key next to a border between two codes goes the other way with an error of fp32 arithmetic, and as often as that error is large.
    # The plain form in fp32, sines and cosines rounded from 64 bits, has a half step of 2^-24 each of two factors, two products and a sum;
    # the kernel has one of the angle more: its codes may differ from the exact ones' some tenths more often.  1.5 times leaves three
    # standard deviations of the counts, some ninety; functions off by 2^-23 are at more than twice.
    import torch
    B, Hkv, n, d, P = 16, 16, 2048, 128, 64
    half = d // 2
    g = torch.Generator(device="cuda").manual_seed(seed)
    K = (1.5 * torch.randn((B, Hkv, n, d), generator=g, device="cuda")).bfloat16()
    f = (500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()
    start = torch.randint(0, 130000, (B,), generator=g, device="cuda") // P * P
    per = (int(start.max()) + n) // P
    pages = B * n // P
    table = torch.zeros((B, per), dtype=torch.int32, device="cuda")
    for b in range(B):
        table[b, int(start[b]) // P:int(start[b]) // P + n // P] = torch.arange(b * (n // P), (b + 1) * (n // P), device="cuda")
    Kc, Vc = (torch.zeros(s, dtype=torch.float8_e4m3fn, device="cuda") for s in ((pages, Hkv, P, d), (pages, Hkv, d, P)))
    ks, vs = torch.ones((pages, Hkv), device="cuda"), torch.ones((pages, Hkv), device="cuda")
    dd.dd_paged_cache_append(Kc, Vc, K, K, table, start.int(), k_scale=ks, v_scale=vs, inv_freq=f)

    def codes(x):                                            # of rows [Hkv, n, d] in the scales that their pages have
        x = x.reshape(Hkv, n // P, P, d) / scale.to(x.dtype)[:, :, None, None]
        return x.to(torch.float64)
    off = {"plain": 0, "kernel": 0}
    for b in range(B):
        scale = ks[b * (n // P):(b + 1) * (n // P)].t()
        a = (start[b] + torch.arange(n, device="cuda")).double()[:, None] * f.double()
        turned = {}
        for t in (torch.float64, torch.float32):
            c, s, u, v = a.cos().to(t), a.sin().to(t), K[b, ..., :half].to(t), K[b, ..., half:].to(t)
            turned[t] = codes(torch.cat([u * c - v * s, v * c + u * s], -1))
        rounded = {t: torch.round(x / step) * step for t, x in turned.items()
                   for step in [torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)]}
        own = Kc[b * (n // P):(b + 1) * (n // P)].transpose(0, 1).double()
        off["plain"] += int((rounded[torch.float32] != rounded[torch.float64]).sum())
        off["kernel"] += int((own != rounded[torch.float64]).sum())
    assert 20 < off["plain"] and off["kernel"] <= 1.5 * off["plain"], off


@pytest.mark.parametrize("d", [64, 128])
def test_fp32_norm(d):
    # In units of 2^-24, relative: the sum of squares goes through two roundings of products, three sums of a lane's and three across lanes at
    # most, 8, of which the root has half, 4; 1/d is exact, the sum with eps 1, halved 0.5; the root's own 1 (half a step, and its correction);
    # times the weight 1, times the root 1: 7.5.  A row of zeros stays zeros, one beside eps is a matter of the sum with it alone.
    import torch
    rng = np.random.default_rng(d)
    x = (rng.standard_normal((1, 2, 4096, d)) * 2.0 ** rng.integers(-30, 30, (1, 2, 4096, 1))).astype(np.float32)
    x[0, 0, :7] = 0
    w = (1 + 0.2 * rng.standard_normal(d)).astype(np.float32)
    for eps in (1e-6, 1.2e-38):
        got, _ = dd.dd_qk_norm_rope(dev(x), q_weight=dev(w), eps=eps)
        y = x.astype(np.float64)
        want = y / np.sqrt((y * y).mean(-1, keepdims=True) + float(np.float32(eps))) * w.astype(np.float64)
        off = np.abs(host(got) - want) - 7.5 * 2.0 ** -24 * np.abs(want)
        assert (off <= 1e-45).all(), f"eps {eps}: {(np.abs(host(got) - want) / np.maximum(np.abs(want), 1e-30)).max() * 2 ** 24:.2f} x 2^-24"
