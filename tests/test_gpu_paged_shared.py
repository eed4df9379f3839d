"""GPU parity of dd_paged_attention_shared against the fp64 oracle, and against dd_paged_attention on tables that repeat the prefixes."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from paper_2604_05250_amd.step import capture_step
from _paged import attention_tolerance, dev, fp8_cache, host, ints, rounded
from test_gpu_guard_bands import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["rule", "0", "1"])
def way(request, monkeypatch):
    """by the library's rule; every prefix for its sequences together; every sequence's prefix and own keys in one go"""
    if request.param != "rule":
        monkeypatch.setenv("DD_TUNE_SHARED_WHOLE", request.param)



def _case(starts, H, Hkv, n, d, P, cache, prefix_lens, lens, per_prefix=None, per=None, seed=0, poison=False, B=None, prefix_table=None, table=None):
    import torch
    rng = np.random.default_rng(seed)
    G, B = len(starts) - 1, B or max(starts)
    pp, po = per_prefix or max(1, max(-(-x // P) for x in prefix_lens)), per or max(1, max(-(-x // P) for x in lens))
    pages = G * pp + B * po + 2
    order = rng.permutation(pages)
    ptable = order[:G * pp].reshape(G, pp).astype(np.int32) if prefix_table is None else np.asarray(prefix_table, np.int32)
    otable = order[G * pp:G * pp + B * po].reshape(B, po).astype(np.int32) if table is None else np.asarray(table, np.int32)
    Q, q64 = rounded(rng.standard_normal((B, H, n, d)), torch.bfloat16)
    if cache == "fp8":
        Kc, kc, ks, ks64 = fp8_cache(rng, (pages, Hkv, P, d), -9, -6)
        Vc, vc, vs, vs64 = fp8_cache(rng, (pages, Hkv, d, P), -9, -6)
    else:
        Kc, kc = rounded(rng.standard_normal((pages, Hkv, P, d)), torch.bfloat16)
        Vc, vc = rounded(rng.standard_normal((pages, Hkv, d, P)), torch.bfloat16)
        ks = vs = ks64 = vs64 = None
    if poison:                                               # slots that hold no position hold NaN
        used = np.zeros((pages, P), bool)
        for t, held, width in ((ptable, prefix_lens, pp), (otable, lens, po)):
            for i in range(len(t)):
                for p in range(min(max(int(held[i]), 0), width * P)):
                    if 0 <= t[i][p // P] < pages:
                        used[t[i][p // P], p % P] = True
        hole = dev(~used)[:, None, :, None]
        if cache == "fp8":
            Kc.view(torch.uint8).masked_fill_(hole, 0x7f)
            Vc.view(torch.uint8).masked_fill_(hole.transpose(2, 3), 0xff)
            ks[dev(~used.any(1))] = float("nan")
            vs[dev(~used.any(1))] = float("nan")
        else:
            Kc.masked_fill_(hole, float("nan"))
            Vc.masked_fill_(hole.transpose(2, 3), float("nan"))
    args = dict(Q=Q, Kc=Kc, Vc=Vc, prefix_table=ints(ptable), prefix_lens=ints(prefix_lens), group_starts=ints(starts), block_table=ints(otable),
                kv_lens=ints(lens), k_scale=ks, v_scale=vs)
    return args, (q64, kc, vc, ks64, vs64, ptable, prefix_lens, starts, otable, lens)


def _check(*a, **kw):
    import torch
    args, o = _case(*a, **kw)
    O = torch.full_like(args["Q"], float("nan"))
    got = dd.dd_paged_attention_shared(**args, O=O)
    torch.cuda.synchronize()
    assert got.data_ptr() == O.data_ptr()
    want, A = paged.paged_attention_shared(*o)
    off = np.abs(host(O) - want) - attention_tolerance(want, A)
    assert (off <= 0).all(), f"{np.count_nonzero(~(off <= 0))} elements off, by up to {np.nanmax(off):.3e}"
    return args, O


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("starts,H,Hkv,n,d,P,prefix_lens,lens", [
    ([0, 1], 1, 1, 1, 64, 16, [1], [1]), ([0, 3], 4, 1, 1, 128, 64, [100], [5, 64, 65]), ([0, 2, 5], 8, 2, 1, 128, 16, [33, 200], [17, 1, 3, 90, 16]),
    ([0, 9], 2, 2, 1, 64, 128, [777], [3] * 9), ([0, 1, 2, 3], 7, 1, 3, 128, 32, [64, 65, 63], [10, 31, 32]), ([0, 40], 8, 4, 1, 128, 64, [130], list(range(1, 41))),
    ([0, 4], 4, 2, 33, 64, 64, [300], [40, 50, 60, 129]), ([0, 2, 2, 3], 4, 4, 16, 128, 16, [50, 7, 81], [16, 17, 40]), ([0, 5], 28, 4, 2, 64, 16, [500], [1, 2, 100, 64, 33])])
def test_parity(cache, starts, H, Hkv, n, d, P, prefix_lens, lens, way):
    _check(starts, H, Hkv, n, d, P, cache, prefix_lens, lens)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("n", [1, 24, 70])
def test_what_no_position_holds_does_not_matter(cache, n, way):
    _check([0, 2, 5], 4, 2, n, 128, 16, cache, [1, 100], [0, 1, 15, 33, 60], per=5, per_prefix=8, poison=True)
    _check([0, 3], 4, 2, n, 64, 128, cache, [129], [127, 129, 0], per=3, per_prefix=4, poison=True)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_empty_prefixes_groups_and_sequences(cache, way):
    # sequence 0 has no group; an empty group; a group without a prefix; lengths out of range; rows without any key get zeros
    _, O = _check([1, 3, 3, 5, 6], 4, 2, 2, 128, 16, cache, [40, 10 ** 9, -5, 10 ** 9], [20, 0, 33, 0, 9, -1, 10 ** 9], per=3, per_prefix=4, poison=True, B=7)
    assert not O[3].any() and all(bool(O[b].any()) for b in (0, 1, 2, 4, 5, 6))


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_pages_that_are_none(cache, way):
    _, O = _check([0, 2, 3], 4, 2, 3, 128, 16, cache, [64, 64], [40, 40, 20], per=3, per_prefix=4, prefix_table=[[0, 99, 1, -1], [-1, 2 ** 31 - 1, -2 ** 31, 14]],
                  table=[[2, 3, 4], [5, -7, 6], [-1, 13, 0]], poison=True)
    assert all(bool(O[b].any()) for b in range(3))           # (sequence 2: its prefix's last page and its own second one are there)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("starts,H,Hkv,n,prefix", [([0, 2], 8, 2, 1, 4097), ([0, 1, 3], 4, 1, 20, 2500), ([0, 12], 8, 2, 1, 3000)])
def test_long_prefixes_are_split(cache, starts, H, Hkv, n, prefix, way):
    B = starts[-1]
    _check(starts, H, Hkv, n, 128, 64, cache, [prefix] + [prefix // 2] * (len(starts) - 2), [(37 * b) % 90 for b in range(B)])


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_long_own_parts_are_split(cache, way):
    _check([0, 2], 4, 1, 1, 128, 64, cache, [70], [1500, 333])


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("d,P", [(64, 16), (64, 128), (128, 32), (128, 64)])
def test_rows_by_the_hundred(cache, d, P, way):
    # two row blocks per workgroup for the prefixes (more than 512 blocks of 32 rows), the own keys' one; groups that end within a tile
    _check([0, 5, 11], 48, 48, 34, d, P, cache, [190, 65], [0, 1, 20, 33, 64, 65, 40, 7, 0, 100, 12], poison=True, seed=d + P)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("d,P", [(64, 32), (128, 128)])
def test_rows_by_the_thousand(cache, d, P, way):
    # four row blocks per workgroup, of the prefix and of the own keys
    _check([0, 9], 94, 47, 64, d, P, cache, [130], [66, 0, 1, 64, 65, 40, 33, 17, 90], poison=True, seed=d + P)


def test_many_groups(way):
    # more groups than a wave has lanes, most of them of one sequence, some of none
    rng = np.random.default_rng(3)
    starts = np.concatenate([[0], np.cumsum(rng.integers(0, 3, 150))])
    _check(starts.tolist(), 4, 2, 1, 64, 16, "bf16", rng.integers(0, 40, 150).tolist(), rng.integers(0, 30, int(starts[-1])).tolist(), per=2, per_prefix=3, poison=True)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("n", [1, 40])
def test_agrees_with_the_call_on_whole_tables(cache, n, way):
    # prefixes of whole pages: the same cache by tables that have the prefix's pages first
    import torch
    B, P = 6, 64
    args, _ = _case([0, 4, 6], 8, 2, n, 128, P, cache, [5 * P, 3 * P], [30, 64, 100, 1, 77, 5], per_prefix=5)
    O = dd.dd_paged_attention_shared(**args)
    whole, lens = [], []
    for b in range(B):
        g = 0 if b < 4 else 1
        k = [5, 3][g]
        whole.append(torch.cat([args["prefix_table"][g, :k], args["block_table"][b], args["block_table"].new_full((5 - k,), -1)]))
        lens.append(k * P + int(args["kv_lens"][b]))
    alone = dd.dd_paged_attention(args["Q"], args["Kc"], args["Vc"], torch.stack(whole), ints(lens), k_scale=args["k_scale"], v_scale=args["v_scale"])
    # either is off by its weights' and its own rounding, 2^-8 and 2^-8 of the values' size at most
    assert bool(((O.float() - alone.float()).abs() <= 4 * 2.0 ** -8 * host_values(args, O)).all())
    again = dd.dd_paged_attention_shared(**args)
    assert torch.equal(O, again)


def host_values(args, O):
    """the largest value that a sequence's output can come from, over its head dims"""
    import torch
    v = args["Vc"].float() if args["v_scale"] is None else args["Vc"].view(torch.float8_e4m3fn).float() * args["v_scale"][..., None, None]
    return v.abs().amax()


def test_starts_that_descend_stay_inside_the_tensors(way):
    import torch
    for n, H in ((1, 8), (40, 48)):
        args, _ = _case([0, 3, 5, 8], H, H // 4, n, 128, 16, "bf16", [100, 40, 60], [20] * 8)
        g = Guarded()
        O = g.empty(tuple(args["Q"].shape), torch.bfloat16)
        need = dd.dd_paged_attention_shared_workspace_bytes(n, 8, H, H // 4, 128, 16, 3, 7, 2, dd.BF16)
        for starts in ([8, 0, 8, 0], [0, 8, 0, 8], [-2 ** 31, 2 ** 31 - 1, -5, 99], [5, 4, 3, 2], [2 ** 31 - 1] * 4, [-1] * 4):
            args["group_starts"].copy_(ints(starts))
            with dd.fixed_workspace(g.empty((need,), torch.uint8)):
                dd.dd_paged_attention_shared(**args, O=O)
            g.check(f"starts {starts}")


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("n,P", [(1, 64), (33, 16), (70, 128)])
def test_nothing_else_is_written(cache, n, P, way):
    import torch
    args, _ = _case([0, 2, 3], 4, 2, n, 128, P, cache, [300, 31], [50, 1, 81])
    kept = {k: v.clone() for k, v in args.items() if v is not None}
    g = Guarded()
    O = g.empty(tuple(args["Q"].shape), torch.bfloat16)
    need = dd.dd_paged_attention_shared_workspace_bytes(n, 3, 4, 2, 128, P, 2, args["prefix_table"].shape[1], args["block_table"].shape[1],
                                                        dd.FP8_E4M3 if cache == "fp8" else dd.BF16)
    with dd.fixed_workspace(guarded_workspace(g, need)):
        dd.dd_paged_attention_shared(**args, O=O)
    g.check(f"{cache} n {n} P {P}")
    assert all(torch.equal(args[k].view(torch.uint8), v.view(torch.uint8)) for k, v in kept.items()) and bool(O.isfinite().all())


@pytest.mark.parametrize("n", [1, 48])
def test_graph_replays_match_eager_calls(n, way):
    import torch
    args, _ = _case([0, 3, 5], 16, 4, n, 128, 64, "fp8", [900, 200], [20, 64, 3, 90, 1], per=2)
    O = torch.zeros_like(args["Q"])
    graph = capture_step(lambda: dd.dd_paged_attention_shared(**args, O=O))
    for rep in range(5):
        args["Q"].copy_(args["Q"].roll(1, 0))
        args["kv_lens"].copy_(args["kv_lens"].roll(1, 0))
        args["prefix_lens"].sub_(7)
        args["group_starts"].copy_(ints([0, 1 + rep % 4, 5]))
        want = dd.dd_paged_attention_shared(**args)
        torch.cuda.synchronize()
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want), f"replay {rep}"


def test_streams_side_by_side(way):
    import torch
    cases = [_case([0, 4], 8, 2, 1, 128, 64, "fp8", [1000 + 300 * k], [20, 64, 3, 90], seed=k)[0] for k in range(3)]
    want = [dd.dd_paged_attention_shared(**c) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [[] for _ in cases]
    for _ in range(5):
        for c, s, to in zip(cases, streams, got):
            with torch.cuda.stream(s):
                to.append(dd.dd_paged_attention_shared(**c))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, bs in zip(want, got) for b in bs)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("n,d", [(1, 128), (5, 64), (40, 128), (200, 64)])
def test_prefix_and_own_keys_in_one_go(cache, P, n, d):
    # short capacities need no workspace: prefixes that end anywhere within a tile or page, no prefix, no keys, pages that are none
    args, o = _case([0, 2, 3, 3, 6], 4, 2, n, d, P, cache, [1, 63, 64, 130], [0, 1, 33, 64, 0, 17], per=-(-64 // P), per_prefix=-(-130 // P), poison=True, B=6, seed=n)
    assert dd.dd_paged_attention_shared_workspace_bytes(n, 6, 4, 2, d, P, 4, -(-130 // P), -(-64 // P), dd.FP8_E4M3 if cache == "fp8" else dd.BF16) == 0
    want, A = paged.paged_attention_shared(*o)
    got = host(dd.dd_paged_attention_shared(**args))
    assert (np.abs(got - want) <= attention_tolerance(want, A)).all()


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("d,P,H,n", [(128, 64, 64, 8), (64, 16, 66, 34), (128, 16, 96, 64)])
def test_full_row_blocks_in_one_go(cache, d, P, H, n):
    # calls whose rows fill row blocks, of one, two and four per workgroup, whatever the capacity
    import torch
    G, B, Hkv = 2, 9, H // 2
    assert (dd.dd_paged_attention_shared_workspace_bytes(n, B, H, Hkv, d, P, G, 4096 // P, 1, dd.FP8_E4M3 if cache == "fp8" else dd.BF16) == 0) == (n != 8)
    _check([0, 4, 9], H, Hkv, n, d, P, cache, [100, 65], [0, 1, 40, 64, 65, 30, 7, 0, 64], poison=True, seed=n)


def test_sequences_without_a_group_in_one_go():
    _, O = _check([2, 3, 3], 4, 2, 3, 128, 16, "bf16", [40, 9], [20, 0, 0, 33], per=3, per_prefix=3, poison=True, B=4)
    assert not O[1].any() and bool(O[2].any()) and bool(O[0].any())


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_more_rows_by_the_thousand(cache, way):
    # four row blocks per workgroup with either type, of whole groups and of sequences
    _check([0, 10], 94, 47, 64, 64, 64, cache, [65], [66, 0, 1, 64, 65, 40, 33, 17, 90, 3], poison=True)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_two_kinds_of_workgroups_in_two_launches(cache, way):
    # many sequences of few rows: the prefix's rows two or four blocks at a time, the own ones one
    rng = np.random.default_rng(2)
    for B, H in ((180, 96), (100, 256)):
        _check([0, B // 3, B], H, H // 2, 1, 64, 32, cache, [70, 33], rng.integers(0, 40, B).tolist(), poison=True)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_offsets_past_32_bits(cache, way):
    # the pages of a small cache, scattered over one of more than 4 GB
    import torch
    args, _ = _case([0, 3, 5], 8, 8, 2, 128, 128, cache, [700, 150], [20, 130, 3, 90, 1])
    pages = args["Kc"].shape[0]
    many = 5 * (1 << 30) // (8 * 128 * 128 * args["Kc"].element_size())
    to = torch.linspace(0, many - 1, pages, device="cuda").long().flip(0)
    big = dict(args)
    for name in ("Kc", "Vc"):
        small = args[name].view(torch.uint8)
        wide = torch.empty((many,) + tuple(small.shape[1:]), dtype=torch.uint8, device="cuda")
        wide[to] = small
        big[name] = wide.view(args[name].dtype)
    for name in ("k_scale", "v_scale"):
        if args[name] is not None:
            big[name] = torch.full((many, 8), float("nan"), device="cuda")
            big[name][to] = args[name]
    for name in ("prefix_table", "block_table"):
        big[name] = to[args[name].long()].int()
    assert torch.equal(dd.dd_paged_attention_shared(**args), dd.dd_paged_attention_shared(**big))
