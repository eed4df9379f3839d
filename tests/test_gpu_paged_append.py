"""GPU parity of dd_paged_cache_append against the fp64 oracle: what is written, the scales, and every byte that is not."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from _paged import E4M3, ROW_FAST, codes_of, dev, fp8_cache, host, ints, rounded

pytestmark = pytest.mark.gpu


def _freq(rot):
    return None if not rot else (10000.0 ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)


def _tables(rng, B, per, pages):
    return rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)


def _check(B, Hkv, n, d, P, cache, starts, rows="bf16", kv_lens=None, n_rows=None, rot=None, norm=True, interleaved=False, fused=True, table=None,
           per=None, scale=1.5, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    t = torch.bfloat16 if rows == "bf16" else torch.float32
    per = per or max(-(-(max(s, 0) + n) // P) for s in starts)
    pages = B * per + 2
    table = _tables(rng, B, per, pages) if table is None else np.asarray(table, np.int32)
    if cache == "fp8":
        Kc, kc, ks, ks64 = fp8_cache(rng, (pages, Hkv, P, d))
        Vc, vc, vs, vs64 = fp8_cache(rng, (pages, Hkv, d, P))
    else:
        Kc, kc = rounded(rng.standard_normal((pages, Hkv, P, d)), torch.bfloat16)
        Vc, vc = rounded(rng.standard_normal((pages, Hkv, d, P)), torch.bfloat16)
        ks = vs = ks64 = vs64 = None
    fresh, _ = rounded(rng.standard_normal((B, n, 2 * Hkv * d)) * scale, t)
    K, V = fresh[..., :Hkv * d].view(B, n, Hkv, d).transpose(1, 2), fresh[..., Hkv * d:].view(B, n, Hkv, d).transpose(1, 2)
    if not fused:
        K, V = K.contiguous(), V.contiguous()
    w, w64 = rounded(1 + 0.2 * rng.standard_normal(d), t) if norm else (None, None)
    f = _freq(d if rot is None else rot)
    before = {k: (codes_of(c) if cache == "fp8" else c.clone()) for k, c in (("K", Kc), ("V", Vc))}
    dd.dd_paged_cache_append(Kc, Vc, K, V, ints(table), ints(starts), kv_lens=None if kv_lens is None else ints(kv_lens),
                             n_rows=None if n_rows is None else ints(n_rows), k_scale=ks, v_scale=vs, k_weight=w, eps=1e-5,
                             inv_freq=None if f is None else dev(f), interleaved=interleaved)
    torch.cuda.synchronize()
    Kn, Vn, ksn, vsn, (Kraw, Vraw) = paged.paged_append(kc, vc, ks64, vs64, host(K), host(V), table, starts, kv_lens, n_rows, w64,
                                                       float(np.float32(1e-5)), f, interleaved)
    # keys carry the arithmetic's error, as a share of their row's largest magnitude before it is rounded; values are exact
    top = np.abs(Kraw).max(-1, keepdims=True)
    for name, got, want, raw, old, err in (("K", Kc, Kn, Kraw, kc, ROW_FAST * top), ("V", Vc, Vn, Vraw, vc, 0.0)):
        if cache == "fp8":
            values = E4M3[codes_of(got)]
            half = paged.e4m3_step(raw) / 2
            same = raw == old                                       # neither written nor in a new scale
            assert np.array_equal(codes_of(got)[same], before[name][same]), f"{name}: a code that stays was changed"
        else:
            values = host(got)
            half = 2.0 ** -8 * np.abs(raw)
            same = raw == old
            assert np.array_equal(values[same], old[same])
        off = np.abs(values - raw) - (half + err * (1 + 2.0 ** -4))
        assert (off <= 0).all(), f"{name}: {np.count_nonzero(off > 0)} elements off by up to {off.max():.3e}"
        if cache == "fp8":                                          # (the oracle leaves the rounding of bf16 pages out)
            assert np.mean(values != want) < 1e-3                   # a result next to a border may go either way, others not
    if cache == "fp8":
        assert np.array_equal(host(ks), ksn) and np.array_equal(host(vs), vsn)
    return Kc, Vc


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("rows", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hkv,n,d,P,starts", [
    (1, 1, 1, 64, 16, [0]), (2, 8, 1, 128, 64, [63, 64]), (3, 2, 33, 128, 16, [5, 0, 47]), (2, 1, 130, 64, 128, [100, 255]),
    (2, 3, 64, 128, 32, [31, 32]), (1, 2, 77, 64, 64, [1])])
def test_parity(cache, rows, B, Hkv, n, d, P, starts):
    _check(B, Hkv, n, d, P, cache, starts, rows)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("kw", [
    dict(norm=False), dict(rot=0), dict(rot=32, interleaved=True), dict(norm=False, rot=0, fused=False), dict(n_rows=[0, 7, 99, -4]),
    dict(kv_lens=[200, 60, 61, 0]), dict(kv_lens=[200, 60, 61, 0], n_rows=[3, 0, 20, 20]), dict(scale=300.0), dict(scale=1e-3, norm=False)])
def test_options(cache, kw):
    # (kv_lens past the rows: a block within the sequence is rewritten)
    _check(4, 2, 20, 64, 32, cache, [40, 60, 11, 64], per=7, **kw)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("d,P", [(128, 128), (64, 128), (128, 64), (64, 32)])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65])
def test_few_rows(cache, d, P, n):
    # at the pages' borders and across them, at the end and within sequences, with rows that are small beside what the pages hold and large
    for scale in (1e-3, 1.5, 300.0):
        _check(4, 3, n, d, P, cache, [P - n, P - 1, 5, 2 * P], rows="f32" if n % 16 == 15 else "bf16", per=4, scale=scale, norm=False, seed=n)
    _check(4, 3, n, d, P, cache, [P - n, P - 1, 5, 2 * P - 3], kv_lens=[4 * P, P + 3, 5, 2 * P + n], per=4, scale=40.0, interleaved=True, seed=n)
    _check(4, 3, n, d, P, cache, [P - n, P - 1, -5, 4 * P - 3], n_rows=[n - 1, 1, n, n], per=4, rot=32, seed=n)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_rows_and_pages_that_are_skipped(cache):
    # positions before the sequence and behind the table, pages that are none, and a start near the type's end
    _check(3, 2, 50, 64, 16, cache, [-7, 30, 2**31 - 20], table=[[0, 99, 2, 3], [4, 5, -1, 7], [8, 9, 10, 11]], per=4)
    _check(2, 1, 9, 64, 16, cache, [-2**31, 60], table=[[0, 1, 2, 3], [4, 5, 6, 7]], per=4, kv_lens=[-5, 2**31 - 1])


def test_scales_that_are_no_power_of_two():
    # pages filled by someone else: a larger scale stays and divides, a smaller one is replaced
    import torch
    rng = np.random.default_rng(8)
    P, d = 32, 64
    Kc, kc, _, _ = fp8_cache(rng, (2, 2, P, d))
    Vc, vc, _, _ = fp8_cache(rng, (2, 2, d, P))
    ks64 = np.array([[0.37, 1.1e-3], [1, 1]], np.float32).astype(np.float64)
    K, k64 = rounded(rng.standard_normal((1, 2, 5, d)), torch.bfloat16)
    ks, vs = dev(ks64.astype(np.float32)), dev(ks64.astype(np.float32))
    dd.dd_paged_cache_append(Kc, Vc, K, K, ints([[0]]), ints([10]), k_scale=ks, v_scale=vs)
    Kn, Vn, ksn, vsn, (Kraw, Vraw) = paged.paged_append(kc, vc, ks64, ks64, k64, k64, [[0]], [10])
    assert np.array_equal(host(ks), ksn) and np.array_equal(host(vs), vsn)
    for got, want, raw in ((Kc, Kn, Kraw), (Vc, Vn, Vraw)):
        # the quotient of scales and its product are rounded to fp32 before the code: 2 steps of 2^-24
        assert (np.abs(E4M3[codes_of(got)] - raw) <= paged.e4m3_step(raw) / 2 + 2.0 ** -22 * np.abs(raw)).all()
        assert np.mean(E4M3[codes_of(got)] != want) < 1e-3


def test_every_code_and_tie_of_values():
    # V is stored without arithmetic: every bf16 number that is a tie or next to one, at a scale of 1
    import torch
    grid = np.unique(np.abs(E4M3[np.isfinite(E4M3)]))
    mid = (grid[1:] + grid[:-1]) / 2
    x = np.concatenate([grid, mid, np.nextafter(mid.astype(np.float32), 0), np.nextafter(mid.astype(np.float32), 1e9)]).astype(np.float32)
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros((-len(x)) % (64 * 16), np.float32)]).reshape(1, 1, -1, 64)
    n = x.shape[2]
    x[0, 0, :, 0] = 448.0                                                    # every page has the scale 1
    Kc = torch.zeros((n // 16, 1, 16, 64), dtype=torch.uint8, device="cuda")
    Vc = torch.zeros((n // 16, 1, 64, 16), dtype=torch.uint8, device="cuda")
    ks, vs = torch.full((n // 16, 1), 7.0, device="cuda"), torch.full((n // 16, 1), 7.0, device="cuda")
    X = dev(x)
    dd.dd_paged_cache_append(Kc, Vc, X, X, ints(np.arange(n // 16)[None]), ints([0]), k_scale=ks, v_scale=vs)
    assert (vs == 1).all() and (ks == 1).all()
    want = paged.e4m3(x[0, 0]).reshape(n // 16, 16, 64)
    assert np.array_equal(E4M3[codes_of(Kc)][:, 0], want) and np.array_equal(E4M3[codes_of(Vc)][:, 0].swapaxes(-1, -2), want)


def test_zero_rows_and_page_after_page():
    # rows of zeros take the least scale and keep their page's; token after token is block at once but for the scales on the way
    import torch
    Kc = torch.zeros((2, 1, 16, 64), dtype=torch.uint8, device="cuda")
    Vc = torch.zeros((2, 1, 64, 16), dtype=torch.uint8, device="cuda")
    ks, vs = torch.full((2, 1), float("nan"), device="cuda"), torch.full((2, 1), float("nan"), device="cuda")
    zero = torch.zeros((1, 1, 3, 64), device="cuda")
    dd.dd_paged_cache_append(Kc, Vc, zero, zero, ints([[1, 0]]), ints([0]), k_scale=ks, v_scale=vs)
    assert ks[1, 0] == 2.0 ** -126 == vs[1, 0] and not Kc.any() and ks[0].isnan()
    rows = (2.0 ** torch.randint(-1, 2, (1, 1, 20, 64), device="cuda").float())
    for r in range(20):
        dd.dd_paged_cache_append(Kc, Vc, rows[:, :, r:r + 1], rows[:, :, r:r + 1], ints([[1, 0]]), ints([3 + r]), k_scale=ks, v_scale=vs)
    got = E4M3[codes_of(Kc)] * host(ks)[..., None, None]
    assert np.array_equal(np.concatenate([got[1, 0], got[0, 0]])[3:23], host(rows)[0, 0]) and not got[1, 0, :3].any()
    got = (E4M3[codes_of(Vc)] * host(vs)[..., None, None]).swapaxes(-1, -2)
    assert np.array_equal(np.concatenate([got[1, 0], got[0, 0]])[3:23], host(rows)[0, 0])


def test_a_row_that_is_not_finite_stays_in_its_page_and_head():
    import torch
    rng = np.random.default_rng(3)
    x, _ = rounded(rng.standard_normal((2, 2, 40, 64)), torch.bfloat16)
    y = x.clone()
    y[0, 1, 20, 3], y[1, 0, 39, 0] = float("inf"), float("nan")             # pages 1 and 2 of their sequences
    table, caches = ints([[0, 1, 2], [3, 4, 5]]), []
    for rows in (x, y):
        Kc, Vc = torch.zeros((6, 2, 16, 64), dtype=torch.uint8, device="cuda"), torch.zeros((6, 2, 64, 16), dtype=torch.uint8, device="cuda")
        ks, vs = torch.ones((6, 2), device="cuda"), torch.ones((6, 2), device="cuda")
        dd.dd_paged_cache_append(Kc, Vc, rows, rows, table, ints([0, 0]), k_scale=ks, v_scale=vs)
        caches.append((Kc, Vc, ks, vs))
    others = torch.ones((6, 2), dtype=torch.bool, device="cuda")
    others[1, 1] = others[5, 0] = False
    for a, b in zip(*caches):
        assert torch.equal(a[others], b[others])
    assert all(s.isfinite().all() and (s > 0).all() for s in caches[1][2:])


def test_no_rows():
    import torch
    Kc = torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    dd.dd_paged_cache_append(Kc, Kc.new_zeros((2, 1, 64, 16)), Kc.new_empty((1, 1, 0, 64)), Kc.new_empty((1, 1, 0, 64)), ints([[0, 1]]), ints([0]))
    assert not Kc.any()
