"""Attention over shared prefixes in forms that a caller may use beside the usual ones: scores that rise or fall from prefix to own keys, a
query row of NaN, any positive scale and scales at the ends of their range, the same call again, several threads."""
import sys
import threading

import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from _paged import E4M3, attention_tolerance, codes_of, dev, host, ints, rounded
from test_gpu_paged_shared import _case, way  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

# starts of the groups, heads, key/value heads, rows, prefix, own: one row block per workgroup, two, four, and keys that are split
FORMS = [([0, 2, 3], 4, 2, 5, 400, 90), ([0, 8], 48, 48, 43, 130, 70), ([0, 5], 100, 50, 125, 100, 70), ([0, 1], 2, 1, 3, 2500, 400)]


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling"])
@pytest.mark.parametrize("starts,H,Hkv,n,prefix,own", FORMS)
def test_scores_that_rise_or_fall_over_the_keys(cache, order, starts, H, Hkv, n, prefix, own, way):
    # up to 40 in either sign, by the sign of a row, from the prefix's first key to the last own one
    import torch
    rng = np.random.default_rng(prefix)
    P, d, B, G = 32, 128, starts[-1], len(starts) - 1
    pp, po, N = -(-prefix // P), -(-own // P), prefix + own
    v = np.sign(rng.standard_normal(d))
    ramp = np.arange(1, N + 1) / N
    if order == "falling":
        ramp = ramp[::-1]
    t = torch.uint8 if cache == "fp8" else torch.bfloat16
    pages = G * pp + B * po
    Kc, Vc = torch.zeros((pages, Hkv, P, d), dtype=t, device="cuda"), torch.zeros((pages, Hkv, d, P), dtype=t, device="cuda")
    ks, vs = (torch.ones((pages, Hkv), device="cuda") for _ in range(2)) if cache == "fp8" else (None, None)
    order_of = rng.permutation(pages)
    ptable, otable = order_of[:G * pp].reshape(G, pp), order_of[G * pp:].reshape(B, po)
    for table, part in ((ptable, ramp[:prefix]), (otable, ramp[prefix:])):
        K, _ = rounded((part[None, None, :, None] * v * 2).repeat(len(table), 0).repeat(Hkv, 1), torch.bfloat16)
        V, _ = rounded(rng.standard_normal((len(table), Hkv, len(part), d)), torch.bfloat16)
        dd.dd_paged_cache_append(Kc, Vc, K, V, ints(table), ints(np.zeros(len(table))), k_scale=ks, v_scale=vs)
    sign = np.where(np.arange(n) % 2 == 0, 1.0, -1.0)[:, None]
    Q, q64 = rounded((sign * v * 40 / (2 * d / np.sqrt(d)))[None, None].repeat(B, 0).repeat(H, 1), torch.bfloat16)
    plens, lens = [prefix] * G, [own] * B
    got = host(dd.dd_paged_attention_shared(Q, Kc, Vc, ints(ptable), ints(plens), ints(starts), ints(otable), ints(lens), k_scale=ks, v_scale=vs))
    values = (lambda c: E4M3[codes_of(c)]) if cache == "fp8" else host
    want, A = paged.paged_attention_shared(q64, values(Kc), values(Vc), None if ks is None else host(ks), None if vs is None else host(vs), ptable, plens, starts, otable, lens)
    # products of one sign whose magnitudes add to 40 (43 where e4m3 rounded up): 140 steps of 2^-24 x 43 x log2 e < 2^-10 of a weight, in O and its divisor
    assert (np.abs(got - want) <= (2.0 ** -8 + 2 * 2.0 ** -10) * A + 2.0 ** -8 * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("starts,H,Hkv,n,prefix,own", FORMS)
def test_a_query_row_of_nan_stays_alone(cache, starts, H, Hkv, n, prefix, own, way):
    # rows of other sequences are in the same row block on the prefix
    import torch
    B, G = starts[-1], len(starts) - 1
    args, _ = _case(starts, H, Hkv, n, 128, 64, cache, [prefix] * G, [own] * B)
    Q2 = args["Q"].clone()
    Q2[B - 1, H - 1, n // 2, 3] = float("nan")
    a = dd.dd_paged_attention_shared(**args)
    b = dd.dd_paged_attention_shared(**dict(args, Q=Q2))
    assert b[B - 1, H - 1, n // 2].isnan().all()
    b[B - 1, H - 1, n // 2] = a[B - 1, H - 1, n // 2]
    assert torch.equal(a, b)


@pytest.mark.parametrize("d,P", [(128, 64), (64, 16)])
@pytest.mark.parametrize("starts,H,Hkv,n,prefix,own", FORMS)
def test_any_positive_scale(starts, H, Hkv, n, prefix, own, d, P, way):
    # significands all over [1, 2), as for dd_paged_attention
    B, G = starts[-1], len(starts) - 1
    args, o = _case(starts, H, Hkv, n, d, P, "fp8", [prefix - 7 * g for g in range(G)], [own - 3 * b for b in range(B)])
    rng = np.random.default_rng(n)
    ks, vs = ((2.0 ** rng.uniform(-9, -7, o[3].shape)).astype(np.float32) for _ in range(2))
    got = host(dd.dd_paged_attention_shared(**dict(args, k_scale=dev(ks), v_scale=dev(vs))))
    want, A = paged.paged_attention_shared(*o[:3], ks.astype(np.float64), vs.astype(np.float64), *o[5:])
    off = np.abs(got - want) - attention_tolerance(want, A)
    assert (off <= 0).all(), f"{np.count_nonzero(~(off <= 0))} elements off, by up to {np.nanmax(off):.3e}"


@pytest.mark.parametrize("e", [-110, -60, 60, 88])
def test_values_at_the_ends_of_the_scales_range(e, way):
    args, o = _case([0, 3], 2, 1, 3, 128, 64, "fp8", [900], [100, 20, 64])
    vs = np.full(o[4].shape, 2.0 ** e)
    got = host(dd.dd_paged_attention_shared(**dict(args, v_scale=dev(vs.astype(np.float32)))))
    want, A = paged.paged_attention_shared(*o[:4], vs, *o[5:])
    assert (np.abs(got - want) <= (attention_tolerance(want, A) - 1e-30)).all()


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("starts,H,Hkv,n,prefix,own", FORMS)
def test_the_same_call_again(cache, starts, H, Hkv, n, prefix, own, way):
    import torch
    args, _ = _case(starts, H, Hkv, n, 128, 64, cache, [prefix] * (len(starts) - 1), [own] * starts[-1])
    first = dd.dd_paged_attention_shared(**args)
    assert all(torch.equal(first, dd.dd_paged_attention_shared(**args)) for _ in range(5))


def test_no_queries():

    args, _ = _case([0, 2], 4, 2, 1, 64, 16, "fp8", [20], [20, 7])
    args["Q"] = args["Q"][:, :, :0].contiguous()
    assert dd.dd_paged_attention_shared(**args).shape == (2, 4, 0, 64)


def test_a_capacity_far_beyond_the_lengths():
    import torch
    args, o = _case([0, 2, 5], 8, 2, 1, 128, 64, "fp8", [700, 90], [100, 3, 0, 64, 65])
    for name, width in (("prefix_table", 3000), ("block_table", 1600)):
        wide = torch.full((len(args[name]), width), -1, dtype=torch.int32, device="cuda")
        wide[:, :args[name].shape[1]] = args[name]
        args[name] = wide
    want, A = paged.paged_attention_shared(*o)
    assert (np.abs(host(dd.dd_paged_attention_shared(**args)) - want) <= attention_tolerance(want, A)).all()


def test_threads_on_one_stream():
    # calls of several launches that hand data over in scratch memory, which threads on one stream share
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    shared, _ = _case([0, 4], 8, 2, 1, 128, 64, "fp8", [3000], [20, 64, 3, 90])
    lv, ld = torch.randn((3, 5, 40000), generator=g, device="cuda"), torch.randn((3, 4, 40000), generator=g, device="cuda")
    tokens, u = torch.randint(0, 40000, (3, 4), generator=g, device="cuda").int(), torch.rand((3, 5), generator=g, device="cuda")
    table, stack = ints(np.full((40, 300), -1)), ints(np.arange(40 * 300))
    free, new = ints([40 * 300]), ints(np.arange(40) * 100)
    zero = ints(np.zeros(40))

    def resize():
        a = dd.dd_paged_resize(table, stack, free, zero, new, 16, 700)     # (700 rows of 40 sequences: two launches)
        dd.dd_paged_resize(table, stack, free, a[0], zero, 16)
        return torch.cat([a[0], a[2].flatten()])

    calls = [lambda: dd.dd_paged_attention_shared(**shared), lambda: torch.cat([x.float().flatten() for x in dd.dd_verify_draft(lv, ld, tokens, u)]), resize]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    got, start = [[] for _ in calls], threading.Barrier(len(calls))

    def work(call, to):
        start.wait()
        for _ in range(60):
            to.append(call())
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=work, args=a) for a in zip(calls, got)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    torch.cuda.synchronize()
    for w, outs in zip(want, got):
        assert len(outs) == 60 and all(torch.equal(w, o) for o in outs)
