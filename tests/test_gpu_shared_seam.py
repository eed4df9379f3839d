"""Where a sequence's own positions meet its prefix: values that are 1 for one position each, so that a head dim of the result is that
position's weight, and one that is left out, taken twice or taken for another shows whole.

A weight over the sum of all: rounded to bf16 (2^-8 of itself at most), over a sum of such (2^-8), the quotient rounded again (2^-8); scores are
fp32 sums of up to 128 products whose magnitudes add to some 30 at most, 2^-11 of the weight and of its divisor each (as in _paged.py)."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from _paged import dev, host, ints, rounded

pytestmark = pytest.mark.gpu

TOLERANCE = 3 * 2.0 ** -8 + 2 * 2.0 ** -11


def marked(starts, H, Hkv, n, d, P, prefix_lens, lens, seed=0):
    """Head dims 0 .. d/2 - 1 stand for positions of the prefixes, the others for own ones: ends, page and tile borders, the rest at random.  All
    numbers are bf16's.  -> (Q, K, V, prefix_table, table), K [pages, Hkv, P, d], V [pages, Hkv, d, P]"""
    rng = np.random.default_rng(seed)
    G, B = len(starts) - 1, starts[-1]
    pp, po = max(1, max(-(-x // P) for x in prefix_lens)), max(1, max(-(-x // P) for x in lens))
    pages = G * pp + B * po + 2
    order = rng.permutation(pages)
    ptable, table = order[:G * pp].reshape(G, pp), order[G * pp:G * pp + B * po].reshape(B, po)
    short = lambda x: (np.asarray(x, np.float32).view(np.uint32) & 0xffff0000).view(np.float32).astype(np.float64)
    Q, K = short(rng.standard_normal((B, H, n, d))), short(rng.standard_normal((pages, Hkv, P, d)))
    V = np.zeros((pages, Hkv, d, P))
    for rows, held, first in ((ptable, prefix_lens, 0), (table, lens, d // 2)):
        for row, count in zip(rows, held):
            ends = [count - 1, 0, count - 2, 1] + [x + s for x in range(16, count, 16) for s in (-1, 0)]
            ends = [x for x in dict.fromkeys(ends) if 0 <= x < count]
            if len(ends) > d // 2:
                ends = ends[:4] + list(rng.permutation(ends[4:])[:d // 2 - 4])
            for i, x in enumerate(ends):
                V[row[x // P], :, first + i, x % P] = 1
    return Q, K, V, ptable, table


def wanted(Q, K, V, ptable, prefix_lens, starts, table, lens):
    return paged.paged_attention_shared(Q, K, V, None, None, ptable, prefix_lens, starts, table, lens)[0]


def close(got, want, calls=1):
    return np.abs(got - want) <= calls * TOLERANCE * want


SIZES = [([0, 4, 6], 8, 2, 1, 128, 64, [320, 192], [30, 64, 100, 1, 77, 5]), ([0, 4, 6], 8, 2, 40, 128, 64, [320, 192], [30, 64, 100, 1, 77, 5]),
         ([0, 3], 4, 2, 1, 64, 16, [16], [1, 17, 40]), ([0, 2, 5], 4, 4, 3, 64, 32, [96, 128], [33, 32, 31, 2, 64]), ([0, 2, 3], 4, 1, 33, 128, 128, [128, 256], [129, 1, 64])]


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("way", ["rule", "0", "1"])
@pytest.mark.parametrize("whole_pages", [True, False])
@pytest.mark.parametrize("size", SIZES)
def test_every_position_has_its_weight(size, whole_pages, way, cache, monkeypatch):
    import torch
    if way != "rule":
        monkeypatch.setenv("DD_TUNE_SHARED_WHOLE", way)
    starts, H, Hkv, n, d, P, prefix_lens, lens = size
    if not whole_pages:
        prefix_lens = [x - 1 - 3 * i for i, x in enumerate(prefix_lens)]
    Q, K, V, ptable, table = marked(starts, H, Hkv, n, d, P, prefix_lens, lens)
    q, _ = rounded(Q, torch.bfloat16)
    if cache == "fp8":
        Kc = dev(K, torch.float32).clamp(-448, 448).to(torch.float8_e4m3fn)
        K = Kc.float().cpu().double().numpy()
        Vc, scale = dev(V, torch.float32).to(torch.float8_e4m3fn), torch.ones(K.shape[:2], device="cuda")
    else:
        Kc, Vc, scale = rounded(K, torch.bfloat16)[0], rounded(V, torch.bfloat16)[0], None
    want = wanted(Q, K, V, ptable, prefix_lens, starts, table, lens)
    got = dd.dd_paged_attention_shared(q, Kc, Vc, ints(ptable), ints(prefix_lens), ints(starts), ints(table), ints(lens), k_scale=scale, v_scale=scale)
    assert (want[..., 0].min() > 0) and (want[..., d // 2].min() > 0)     # (the last position of the prefix, the last of its own)
    assert close(host(got), want).all(), np.argwhere(~close(host(got), want))[:8]
    if whole_pages:                                          # the same by tables that have the prefix's pages first
        of = np.searchsorted(starts, np.arange(len(lens)), side="right") - 1
        pages = [x // P for x in prefix_lens]
        rows = [list(ptable[g][:pages[g]]) + list(table[b]) + [-1] * (max(pages) - pages[g]) for b, g in enumerate(of)]
        alone = dd.dd_paged_attention(q, Kc, Vc, ints(rows), ints([prefix_lens[g] + lens[b] for b, g in enumerate(of)]), k_scale=scale, v_scale=scale)
        assert close(host(alone), want).all() and (np.abs(host(got) - host(alone)) <= 2 * TOLERANCE * want).all()
