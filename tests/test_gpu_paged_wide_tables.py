"""Sequences that are short for their table: shared out over workgroups by their own lengths, as a table of just their width would be."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from _paged import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("B,n,held,wide", [(4, 64, [2048, 2047, 1030, 1], 8192), (3, 64, [2048, 2000, 64], 16384), (6, 33, [1300, 2048, 5, 64, 0, 1999], 4096)])
def test_short_sequences_of_many_rows_are_not_split(cache, B, n, held, wide):
    # as many row blocks as compute units, or nearly: a second round of workgroups pays for long shares only
    import torch
    rng = np.random.default_rng(B)
    H, Hkv, d, P = 32, 8, 128, 64
    tag = dd.FP8_E4M3 if cache == "fp8" else dd.BF16
    per = 2048 // P
    table = rng.permutation(B * per).reshape(B, per)
    g = torch.Generator(device="cuda").manual_seed(B)
    Kc, Vc = torch.randn((B * per, Hkv, P, d), generator=g, device="cuda"), torch.randn((B * per, Hkv, d, P), generator=g, device="cuda")
    Kc, Vc = (x.to(torch.float8_e4m3fn if cache == "fp8" else torch.bfloat16) for x in (Kc, Vc))
    ks, vs = (torch.ones((B * per, Hkv), device="cuda") if cache == "fp8" else None for _ in range(2))
    Q = torch.randn((B, H, n, d), generator=g, device="cuda").bfloat16()
    spread = np.full((B, wide // P), -1)
    spread[:, :per] = table
    assert dd.dd_paged_attention_workspace_bytes(n, B, H, Hkv, d, P, per, tag) == 0 < dd.dd_paged_attention_workspace_bytes(n, B, H, Hkv, d, P, wide // P, tag)
    a, b = (dd.dd_paged_attention(Q, Kc, Vc, ints(t), ints(held), k_scale=ks, v_scale=vs) for t in (table, spread))
    assert torch.equal(a, b)                                 # the same sums in the same order
