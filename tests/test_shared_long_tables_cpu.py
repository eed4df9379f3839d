"""Attention over shared prefixes in one go (no workspace) counts a sequence's prefix and own positions together in 32 bits: only tables whose
positions leave that room together are taken so, whatever the rule or a hook would choose."""
import pytest

import paper_2604_05250_amd as dd

ROWS = dict(n=64, B=16, H=32, Hkv=8, d=128)                  # rows that fill 1024 row blocks: one go at any ordinary length
MOST = (1 << 30) // 16 - 1                                   # pages of 16 of one table: the largest that the call takes


def _workspace(prefix_pages, pages, page_size=16, cache=dd.FP8_E4M3, G=1):
    r = ROWS
    return dd.dd_paged_attention_shared_workspace_bytes(r["n"], r["B"], r["H"], r["Hkv"], r["d"], page_size, G, prefix_pages, pages, cache)


@pytest.fixture(params=["rule", "1"])
def way(request, monkeypatch):
    if request.param != "rule":
        monkeypatch.setenv("DD_TUNE_SHARED_WHOLE", request.param)


@pytest.mark.parametrize("cache", [dd.BF16, dd.FP8_E4M3])
def test_long_tables_are_taken_in_one_go_while_their_sum_is_small(way, cache):
    for prefix, own in ((128, 16), (2048, 256), (MOST // 2, MOST // 2)):
        assert _workspace(prefix, own, cache=cache) == 0, (prefix, own)


@pytest.mark.parametrize("cache", [dd.BF16, dd.FP8_E4M3])
@pytest.mark.parametrize("G", [1, 3])
def test_tables_of_2_to_30_positions_together_are_not(way, cache, G):
    rows = ROWS["B"] * ROWS["H"] * ROWS["n"]
    for prefix, own in ((MOST, MOST), (MOST, 1), (1, MOST), ((MOST + 1) // 2, (MOST + 1) // 2)):
        # states of a prefix and of own keys at the least: d sums, a reference and a sum of weights each
        assert _workspace(prefix, own, cache=cache, G=G) >= rows * 2 * (ROWS["d"] + 2) * 4, (prefix, own)
    for page_size in (32, 64, 128):
        most = (1 << 30) // page_size - 1
        assert _workspace(most, most, page_size, cache, G) > 0
