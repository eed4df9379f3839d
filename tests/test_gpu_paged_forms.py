"""The paged calls in forms that a caller may use beside the usual ones: scales that are no powers of two and scales at the ends of their
range, batch entries, heads and rows by themselves, the same call again, rotation in place where a workgroup goes through many heads."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from _paged import E4M3, assert_rows, attention_tolerance, codes_of, dev, host, ints, rounded, ROW_F32, ROW_FAST

pytestmark = pytest.mark.gpu

# batch, heads, key/value heads, rows, positions: one row block per workgroup, two, four, and keys that are split
FORMS = [(2, 4, 2, 5, 700), (6, 48, 48, 43, 260), (5, 92, 46, 125, 200), (1, 2, 1, 3, 3000)]


def _fp8(B, H, Hkv, n, N, d, P, scales, seed):
    """numbers of the order of one, whatever the scales: (call's arguments, k_scale, v_scale, table)"""
    import torch
    rng = np.random.default_rng(seed)
    per = -(-N // P)
    pages = B * per + 1
    table = rng.permutation(pages)[:B * per].reshape(B, per)
    codes = rng.integers(0, 256, (2, pages, Hkv, P, d), dtype=np.uint8)
    codes[(codes & 0x7f) == 0x7f] = 0x38
    ks, vs = scales(rng, (pages, Hkv)).astype(np.float32), scales(rng, (pages, Hkv)).astype(np.float32)
    Kc, Vc = dev(codes[0]).view(torch.float8_e4m3fn), dev(np.ascontiguousarray(codes[1].swapaxes(-1, -2))).view(torch.float8_e4m3fn)
    Q, q64 = rounded(rng.standard_normal((B, H, n, d)), torch.bfloat16)
    return Q, q64, Kc, Vc, ks, vs, table


@pytest.mark.parametrize("d,P", [(128, 64), (128, 16), (64, 128), (64, 32)])
@pytest.mark.parametrize("B,H,Hkv,n,N", FORMS)
def test_any_positive_scale(B, H, Hkv, n, N, d, P):
    # significands all over [1, 2): that of k_scale is in the exponent's factor (a product more among the 140 steps), that of v_scale in
    # the weights, as its logarithm (off by 2^-22) and its reciprocal (2^-23): 140 + 1 steps of 2^-24 x 45 + 2^-21 < 2^-11
    Q, q64, Kc, Vc, ks, vs, table = _fp8(B, H, Hkv, n, N, d, P, lambda rng, s: 2.0 ** rng.uniform(-9, -7, s), seed=N + d)
    lens = [N - 37 * b for b in range(B)]
    got = host(dd.dd_paged_attention(Q, Kc, Vc, ints(table), ints(lens), k_scale=dev(ks), v_scale=dev(vs)))
    want, A = paged.paged_attention(q64, E4M3[codes_of(Kc)], E4M3[codes_of(Vc)], ks, vs, table, lens)
    off = np.abs(got - want) - attention_tolerance(want, A)
    assert (off <= 0).all(), f"{np.count_nonzero(~(off <= 0))} elements off, by up to {np.nanmax(off):.3e}"


@pytest.mark.parametrize("e", [-110, -60, 60, 88])
def test_values_at_the_ends_of_the_scales_range(e):
    # a thousand keys of nearly equal weight: no partial sum leaves fp32's range
    Q, q64, Kc, Vc, ks, vs, table = _fp8(1, 2, 1, 3, 1000, 128, 64, lambda rng, s: 2.0 ** rng.uniform(-9, -7, s), seed=1)
    vs[:] = 2.0 ** e
    got = host(dd.dd_paged_attention(Q, Kc, Vc, ints(table), ints([1000]), k_scale=dev(ks), v_scale=dev(vs)))
    want, A = paged.paged_attention(q64, E4M3[codes_of(Kc)], E4M3[codes_of(Vc)], ks, vs, table, [1000])
    assert (np.abs(got - want) <= (attention_tolerance(want, A) - 1e-30)).all()


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_batch_entries_heads_and_rows_alone(cache):
    # (few enough that every call has the same plan, and each row the same sums)
    import torch
    B, H, Hkv, n, N = 3, 8, 2, 17, 900
    Q, _, Kc, Vc, ks, vs, table = _fp8(B, H, Hkv, n, N, 128, 64, lambda rng, s: 2.0 ** rng.uniform(-9, -7, s), seed=5)
    ks, vs = dev(ks), dev(vs)
    if cache == "bf16":
        Kc, Vc, ks, vs = (Kc.float() / 64).bfloat16(), (Vc.float() / 64).bfloat16(), None, None
    held, table = ints([900, 64, 333]), ints(table)
    whole = dd.dd_paged_attention(Q, Kc, Vc, table, held, k_scale=ks, v_scale=vs)
    for b in range(B):
        one = dd.dd_paged_attention(Q[b:b + 1], Kc, Vc, table[b:b + 1], held[b:b + 1], k_scale=ks, v_scale=vs)
        assert torch.equal(one, whole[b:b + 1]), b
    of = (lambda s, g: None if s is None else s[:, g:g + 1].contiguous())
    for g in range(Hkv):
        heads = slice(4 * g, 4 * g + 4)
        one = dd.dd_paged_attention(Q[:, heads].contiguous(), Kc[:, g:g + 1].contiguous(), Vc[:, g:g + 1].contiguous(), table, held, k_scale=of(ks, g),
                                    v_scale=of(vs, g))
        assert torch.equal(one, whole[:, heads]), g
    for i in (0, 8, 16):
        one = dd.dd_paged_attention(Q[:, :, i:i + 1].contiguous(), Kc, Vc, table, held, k_scale=ks, v_scale=vs)
        assert torch.equal(one, whole[:, :, i:i + 1]), i


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,n,N", FORMS)
def test_the_same_call_again(cache, B, H, Hkv, n, N):
    import torch
    Q, _, Kc, Vc, ks, vs, table = _fp8(B, H, Hkv, n, N, 128, 64, lambda rng, s: 2.0 ** rng.uniform(-9, -7, s), seed=6)
    ks, vs = dev(ks), dev(vs)
    if cache == "bf16":
        Kc, Vc, ks, vs = (Kc.float() / 64).bfloat16(), (Vc.float() / 64).bfloat16(), None, None
    call = lambda: dd.dd_paged_attention(Q, Kc, Vc, ints(table), ints([N] * B), k_scale=ks, v_scale=vs)
    first = call()
    assert all(torch.equal(first, call()) for _ in range(5))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_in_place_through_many_heads(dtype, d, interleaved):
    # so many tokens that a workgroup goes through five heads or more, none a multiple of the heads that it has on their way
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(d)
    Q, K = (torch.randn((8, h, 2100, d), generator=g, device="cuda").to(t) for h in (7, 3))
    w = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(t)
    f = dev((10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32))
    kw = dict(q_weight=w, k_weight=w, inv_freq=f, interleaved=interleaved)
    at = [0, 1, 31, 32, 2098, 2099]
    q64 = host(Q[:1, :, at])
    want = dd.dd_qk_norm_rope(Q, K, **kw)
    dd.dd_qk_norm_rope(Q, K, Qo=Q, Ko=K, **kw)
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1])
    assert_rows(host(Q[:1, :, at]), paged.norm_rope(q64, host(w), float(np.float32(1e-6)), host(f), [at], interleaved), 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24,
                ROW_FAST if dtype == "bf16" else ROW_F32)
