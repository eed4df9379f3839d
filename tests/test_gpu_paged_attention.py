"""GPU parity of dd_paged_attention against the fp64 oracle."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from _paged import attention_tolerance, codes_of, dev, fp8_cache, host, ints, rounded

pytestmark = pytest.mark.gpu


def _case(B, H, Hkv, n, d, P, cache, lens, per=None, seed=0, table=None, poison=False, q_scale=1.0):
    import torch
    rng = np.random.default_rng(seed)
    per = per or max(1, max(-(-x // P) for x in lens))
    pages = B * per + 2
    table = rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32) if table is None else np.asarray(table, np.int32)
    Q, q64 = rounded(rng.standard_normal((B, H, n, d)) * q_scale, torch.bfloat16)
    if cache == "fp8":
        Kc, kc, ks, ks64 = fp8_cache(rng, (pages, Hkv, P, d), -9, -6)         # numbers of the order of one
        Vc, vc, vs, vs64 = fp8_cache(rng, (pages, Hkv, d, P), -9, -6)
    else:
        Kc, kc = rounded(rng.standard_normal((pages, Hkv, P, d)), torch.bfloat16)
        Vc, vc = rounded(rng.standard_normal((pages, Hkv, d, P)), torch.bfloat16)
        ks = vs = ks64 = vs64 = None
    if poison:                                                               # slots that hold no position hold NaN
        used = np.zeros((pages, P), bool)
        for b in range(B):
            for p in range(min(max(lens[b], 0), per * P)):
                if 0 <= table[b][p // P] < pages:
                    used[table[b][p // P], p % P] = True
        hole = dev(~used)[:, None, :, None]
        if cache == "fp8":
            Kc.view(torch.uint8).masked_fill_(hole, 0x7f)
            Vc.view(torch.uint8).masked_fill_(hole.transpose(2, 3), 0xff)
            ks[dev(~used.any(1))] = float("nan")
            vs[dev(~used.any(1))] = float("nan")
        else:
            Kc.masked_fill_(hole, float("nan"))
            Vc.masked_fill_(hole.transpose(2, 3), float("nan"))
    return (Q, Kc, Vc, ints(table), ints(lens), ks, vs), (q64, kc, vc, ks64, vs64, table, lens)


def _check(*a, **kw):
    import torch
    (Q, Kc, Vc, table, lens, ks, vs), o = _case(*a, **kw)
    O = torch.full_like(Q, float("nan"))
    got = dd.dd_paged_attention(Q, Kc, Vc, table, lens, k_scale=ks, v_scale=vs, O=O)
    torch.cuda.synchronize()
    assert got.data_ptr() == O.data_ptr()
    want, A = paged.paged_attention(*o)
    off = np.abs(host(O) - want) - attention_tolerance(want, A)
    assert (off <= 0).all(), f"{np.count_nonzero(~(off <= 0))} elements off, by up to {np.nanmax(off):.3e}"
    return O


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,n,d,P,lens", [
    (1, 1, 1, 1, 64, 16, [1]), (1, 4, 1, 1, 128, 64, [512]), (2, 8, 2, 1, 128, 16, [17, 300]), (3, 4, 4, 16, 128, 32, [64, 65, 63]),
    (2, 8, 2, 8, 64, 128, [129, 1000]), (1, 2, 2, 33, 128, 64, [777]), (2, 8, 1, 9, 128, 64, [130, 4]), (1, 7, 1, 32, 64, 16, [250]),
    (1, 2, 1, 200, 128, 32, [333]), (4, 3, 3, 5, 128, 64, [0, 1, 64, 200])])
def test_parity(cache, B, H, Hkv, n, d, P, lens):
    _check(B, H, Hkv, n, d, P, cache, lens)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("n", [1, 24, 70])
def test_what_no_position_holds_does_not_matter(cache, n):
    _check(5, 4, 2, n, 128, 16, cache, [0, 1, 15, 33, 200], per=13, poison=True)
    _check(2, 4, 2, n, 64, 128, cache, [127, 129], per=3, poison=True)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_empty_rows_and_pages_that_are_none(cache):
    # lengths out of range are clamped, pages that are none take no part, a sequence without any key gets zeros
    O = _check(4, 4, 2, 3, 128, 16, cache, [-3, 10**9, 40, 64], per=4,
               table=[[0, 1, 2, 3], [4, 5, 6, 7], [99, 8, -1, 9], [-1, 2**31 - 1, -2**31, 18]], poison=True)
    assert not O[0].any() and not O[3].any() and O[1].any() and O[2].any()


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,n", [(1, 8, 2, 1), (2, 4, 1, 20), (1, 2, 2, 100)])
def test_long_sequences_are_split(cache, B, H, Hkv, n):
    lens = [4097, 70][:B]
    assert dd.dd_paged_attention_workspace_bytes(n, B, H, Hkv, 128, 64, 65, dd.FP8_E4M3) > 0
    _check(B, H, Hkv, n, 128, 64, cache, lens)


@pytest.mark.parametrize("d,P", [(64, 16), (64, 128), (128, 32), (128, 64)])
@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_many_row_blocks(cache, d, P):
    # more than 512 blocks of 32 rows, every one of them short of a whole one: lengths around a tile's and a page's end, and none
    _check(6, 48, 48, 43, d, P, cache, [0, 1, 63, 64, 65, 200], per=-(-200 // P), poison=True, seed=d + P)


@pytest.mark.parametrize("d,P", [(64, 32), (64, 16), (128, 128), (128, 16)])
@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_many_more_row_blocks(cache, d, P):
    # 250 rows of each of 230 key/value heads, 1840 blocks of which every eighth is short of a whole one
    _check(5, 92, 46, 125, d, P, cache, [0, 1, 65, 128, 190], per=-(-190 // P), poison=True, seed=d + P)


@pytest.mark.parametrize("n,lens", [(43, [4096, 130]), (33, [4095, 0])])
def test_many_row_blocks_and_splits(n, lens):
    # the pages of a long sequence are some few that recur: what its table says counts, not which page it is
    rng = np.random.default_rng(n)
    assert dd.dd_paged_attention_workspace_bytes(n, 2, 70, 70, 64, 128, 32, dd.BF16) > 0
    _check(2, 70, 70, n, 64, 128, "bf16", lens, per=32, table=rng.integers(0, 12, (2, 32)))


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("n", [2, 40])
def test_lengths_around_the_splits_ends(cache, n):
    # a capacity of 2304 positions, sequences whose shares end exactly at a split's end, one key before it and one behind it
    lens = [2304, 2303, 256, 255, 257, 513, 1024, 1]
    assert dd.dd_paged_attention_workspace_bytes(n, len(lens), 2, 1, 128, 32, 72, dd.FP8_E4M3) > 0
    _check(len(lens), 2, 1, n, 128, 32, cache, lens, per=72)


def test_capacity_beyond_the_lengths():
    # a table for 100000 positions, sequences of a few: shared out by their own lengths
    (Q, Kc, Vc, table, lens, ks, vs), o = _case(2, 8, 2, 1, 128, 64, "fp8", [100, 700], per=11)
    import torch
    wide = torch.full((2, 1600), -1, dtype=torch.int32, device="cuda")
    wide[:, :11] = table
    got = dd.dd_paged_attention(Q, Kc, Vc, wide, lens, k_scale=ks, v_scale=vs)
    want, A = paged.paged_attention(*o)
    assert (np.abs(host(got) - want) <= attention_tolerance(want, A)).all()


def test_sharp_and_large_scores():
    # one key far above the others, first or last; a query row of NaN stays alone
    import torch
    (Q, Kc, Vc, table, lens, _, _), (q64, kc, vc, _, _, tab, ln) = _case(1, 1, 1, 40, 128, 32, "bf16", [500])
    for key in (0, 63, 64, 499):
        kc2 = kc.copy()
        kc2[tab[0][key // 32], 0, key % 32] = q64[0, 0, 7] * 4
        K2, kc2 = rounded(kc2, torch.bfloat16)
        got = host(dd.dd_paged_attention(Q, K2, Vc, table, lens))
        want, A = paged.paged_attention(q64, kc2, vc, None, None, tab, ln)
        assert (np.abs(got - want) <= attention_tolerance(want, A)).all()
    Q2 = Q.clone()
    Q2[0, 0, 5] = float("nan")
    a, b = dd.dd_paged_attention(Q, Kc, Vc, table, lens), dd.dd_paged_attention(Q2, Kc, Vc, table, lens)
    rest = [i for i in range(40) if i != 5]
    assert b[0, 0, 5].isnan().all() and torch.equal(a[0, 0, rest], b[0, 0, rest])


# batch, heads, key/value heads, rows, positions: one row block per workgroup, two, four, and keys that are split
FORMS = [(2, 4, 2, 5, 700), (6, 48, 48, 43, 260), (5, 92, 46, 125, 200), (1, 2, 1, 3, 3000)]


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling"])
@pytest.mark.parametrize("B,H,Hkv,n,N", FORMS)
def test_scores_that_rise_or_fall_over_the_keys(cache, order, B, H, Hkv, n, N):
    # the largest score so far grows from tile to tile, or all that follows is small: up to 40 in either sign, by the sign of a row
    import torch
    rng = np.random.default_rng(N)
    P, d = 32, 128
    per = -(-N // P)
    v = np.sign(rng.standard_normal(d))
    ramp = np.arange(1, N + 1) / N
    if order == "falling":
        ramp = ramp[::-1]
    K, _ = rounded((ramp[None, None, :, None] * v * 2).repeat(B, 0).repeat(Hkv, 1), torch.bfloat16)
    V, _ = rounded(rng.standard_normal((B, Hkv, N, d)), torch.bfloat16)
    sign = np.where(np.arange(n) % 2 == 0, 1.0, -1.0)[:, None]
    Q, q64 = rounded((sign * v * 40 / (2 * d / np.sqrt(d)))[None, None].repeat(B, 0).repeat(H, 1), torch.bfloat16)
    t = torch.uint8 if cache == "fp8" else torch.bfloat16
    Kc, Vc = torch.zeros((B * per, Hkv, P, d), dtype=t, device="cuda"), torch.zeros((B * per, Hkv, d, P), dtype=t, device="cuda")
    ks, vs = (torch.ones((B * per, Hkv), device="cuda") for _ in range(2)) if cache == "fp8" else (None, None)
    table = rng.permutation(B * per).reshape(B, per)
    dd.dd_paged_cache_append(Kc, Vc, K, V, ints(table), ints(np.zeros(B)), k_scale=ks, v_scale=vs)
    got = host(dd.dd_paged_attention(Q, Kc, Vc, ints(table), ints(np.full(B, N)), k_scale=ks, v_scale=vs))
    from _paged import E4M3
    values = (lambda c: E4M3[codes_of(c)]) if cache == "fp8" else host
    want, A = paged.paged_attention(q64, values(Kc), values(Vc), None if ks is None else host(ks), None if vs is None else host(vs), table, [N] * B)
    # products of one sign whose magnitudes add to 40 (43 where e4m3 rounded up): 140 steps of 2^-24 x 43 x log2 e < 2^-10 of a weight, in O and its divisor
    assert (np.abs(got - want) <= (2.0 ** -8 + 2 * 2.0 ** -10) * A + 2.0 ** -8 * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,n,N", FORMS)
def test_a_query_row_of_nan_stays_alone(cache, B, H, Hkv, n, N):
    import torch
    (Q, Kc, Vc, table, lens, ks, vs), _ = _case(B, H, Hkv, n, 128, 64, cache, [N] * B)
    Q2 = Q.clone()
    Q2[B - 1, H - 1, n // 2, 3] = float("nan")
    a, b = (dd.dd_paged_attention(q, Kc, Vc, table, lens, k_scale=ks, v_scale=vs) for q in (Q, Q2))
    assert b[B - 1, H - 1, n // 2].isnan().all()
    b[B - 1, H - 1, n // 2] = a[B - 1, H - 1, n // 2]
    assert torch.equal(a, b)


def test_no_queries():
    import torch
    (Q, Kc, Vc, table, lens, ks, vs), _ = _case(2, 4, 2, 1, 64, 16, "fp8", [20, 7])
    assert dd.dd_paged_attention(Q[:, :, :0].contiguous(), Kc, Vc, table, lens, k_scale=ks, v_scale=vs).shape == (2, 4, 0, 64)


def test_scales_far_apart():
    # one page's values are 2^40 times the others': weights keep their range
    import torch
    (Q, Kc, Vc, table, lens, ks, vs), o = _case(1, 2, 1, 4, 64, 16, "fp8", [90])
    for factor in (2.0 ** 40, 2.0 ** -40):
        v2 = vs.clone()
        v2[table[0, 1]] *= factor
        got = host(dd.dd_paged_attention(Q, Kc, Vc, table, lens, k_scale=ks, v_scale=v2))
        want, A = paged.paged_attention(*o[:4], host(v2), *o[5:])
        assert (np.abs(got - want) <= attention_tolerance(want, A)).all()


def test_same_bits_again_and_rows_of_heads_alone():
    import torch
    (Q, Kc, Vc, table, lens, ks, vs), _ = _case(3, 8, 2, 17, 128, 64, "fp8", [900, 64, 333])
    a = dd.dd_paged_attention(Q, Kc, Vc, table, lens, k_scale=ks, v_scale=vs)
    for _ in range(3):
        assert torch.equal(a, dd.dd_paged_attention(Q, Kc, Vc, table, lens, k_scale=ks, v_scale=vs))


def test_pages_past_32_bits():
    # a pool of 4.6 GB: pages whose bytes begin past 2^32
    import torch
    pages, Hkv, P, d = 280000, 1, 128, 128
    Kc = torch.zeros((pages, Hkv, P, d), dtype=torch.uint8, device="cuda")
    Vc = torch.zeros((pages, Hkv, d, P), dtype=torch.uint8, device="cuda")
    ks, vs = torch.ones((pages, Hkv), device="cuda"), torch.ones((pages, Hkv), device="cuda")
    rng = np.random.default_rng(9)
    x, x64 = rounded(rng.standard_normal((1, 1, 200, d)), torch.bfloat16)
    table = ints([[pages - 1, pages - 2]])
    dd.dd_paged_cache_append(Kc, Vc, x, x, table, ints([0]), k_scale=ks, v_scale=vs)
    got = host(dd.dd_paged_attention(x[:, :, :3].contiguous(), Kc, Vc, table, ints([200]), k_scale=ks, v_scale=vs))
    tail = slice(pages - 2, pages)
    from _paged import E4M3
    want, A = paged.paged_attention(x64[:, :, :3], E4M3[codes_of(Kc[tail])], E4M3[codes_of(Vc[tail])], host(ks[tail]), host(vs[tail]), [[1, 0]], [200])
    assert (np.abs(got - want) <= attention_tolerance(want, A)).all()
