"""Scales of a paged cache share memory with nothing that their call writes: decided on the host (addresses that are never
dereferenced)."""
import pytest

import paper_2604_05250_amd as dd

SHAPE, PAGES, HKV, P, D, N, B = -2, 9, 2, 16, 64, 5, 2
CACHE, SCALES, ROWS = PAGES * HKV * P * D, PAGES * HKV * 4, B * HKV * N * D * 2
at = {name: (i + 1) << 20 for i, name in enumerate(("Kc", "Vc", "K", "V", "ks", "vs", "Q", "O"))}


def append(**kw):
    a = dict(at, **kw)
    st = (HKV * N * D, N * D, D)
    return dd.lib().dd_paged_cache_append(a["Kc"], a["Vc"], a["ks"], a["vs"], a["K"], *st, a["V"], *st, 64 << 20, 65 << 20, None, None, None, 1e-6, None, 0, 0,
                                          N, B, HKV, D, PAGES, P, 4, dd.BF16, dd.FP8_E4M3, None)


@pytest.mark.parametrize("kw", [
    dict(vs=at["ks"]), dict(vs=at["ks"] + SCALES - 4), dict(ks=at["vs"] + SCALES - 4),
    *[{scale: at[other] + size - 4} for scale in ("ks", "vs") for other, size in (("Kc", CACHE), ("Vc", CACHE), ("K", ROWS), ("V", ROWS))],
    *[{scale: at[other] - SCALES + 4} for scale in ("ks", "vs") for other in ("Kc", "Vc", "K", "V")]])
def test_append_refuses(kw):
    assert append(**kw) == SHAPE


@pytest.mark.parametrize("scale", ["ks", "vs"])
@pytest.mark.parametrize("off", [0, 8 * 3 * D * 2 * B - 4, 4 - SCALES])
def test_attention_refuses_its_output_over_scales(scale, off):
    a = dict(at, **{scale: at["O"] + off})
    assert dd.lib().dd_paged_attention(a["Q"], a["Kc"], a["Vc"], a["ks"], a["vs"], 64 << 20, 65 << 20, a["O"], 3, B, 8, HKV, D, PAGES, P, 4, dd.FP8_E4M3, None, 0,
                                       None) == SHAPE
