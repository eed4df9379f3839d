"""GPU parity of dd_qk_norm_rope against the fp64 oracle."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from _paged import ROW_F32, ROW_FAST, assert_rows, dev, host, ints, rounded

pytestmark = pytest.mark.gpu


def _types(name):
    import torch
    return (torch.bfloat16, 2.0 ** -8, ROW_FAST) if name == "bf16" else (torch.float32, 2.0 ** -24, ROW_F32)


def _freq(rot, theta=10000.0):
    return None if not rot else (theta ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)


def _check(B, H, Hkv, n, d, dtype, rot, norm, interleaved, far=1000, fused=True, positions=True, seed=0):
    import torch
    t, half_step, row = _types(dtype)
    rng = np.random.default_rng(seed)
    rows, _ = rounded(rng.standard_normal((B, n, (H + 2 * Hkv) * d)) * 2, t)
    Q = rows[..., :H * d].view(B, n, H, d).transpose(1, 2)
    K = rows[..., H * d:(H + Hkv) * d].view(B, n, Hkv, d).transpose(1, 2)
    if not fused:
        Q, K = Q.contiguous(), K.contiguous()
    qw, qw64 = rounded(1 + 0.2 * rng.standard_normal(d), t) if norm else (None, None)
    kw, kw64 = rounded(1 + 0.2 * rng.standard_normal(d), t) if norm else (None, None)
    f = _freq(rot)
    pos = rng.integers(0, far, (B, n)) if positions else np.broadcast_to(np.arange(n), (B, n))
    Qo, Ko = dd.dd_qk_norm_rope(Q, K, q_weight=qw, k_weight=kw, eps=1e-5, inv_freq=None if f is None else dev(f),
                                positions=ints(pos) if positions else None, interleaved=interleaved)
    torch.cuda.synchronize()
    assert Qo.shape == (B, H, n, d) and Ko.shape == (B, Hkv, n, d) and Qo.dtype == t and Qo.is_contiguous()
    for got, x, w in ((Qo, Q, qw64), (Ko, K, kw64)):
        assert_rows(host(got), paged.norm_rope(host(x), w, float(np.float32(1e-5)), f, pos, interleaved), half_step, row)
    return Q, K, Qo, Ko


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,n,d,rot,norm,interleaved", [
    (1, 1, 1, 1, 64, 64, True, False), (1, 32, 8, 1, 128, 128, True, False), (2, 4, 2, 33, 64, 32, True, True), (3, 7, 1, 5, 128, 16, True, False),
    (2, 3, 3, 65, 128, 0, True, False), (2, 5, 2, 17, 64, 48, False, True), (1, 2, 1, 31, 128, 112, True, True), (2, 4, 4, 16, 128, 128, False, False)])
def test_parity(dtype, B, H, Hkv, n, d, rot, norm, interleaved):
    _check(B, H, Hkv, n, d, dtype, rot, norm, interleaved)


@pytest.mark.parametrize("which", ["queries", "keys"])
def test_one_side_is_normed(which):
    # the other side's rows are rotated as they are, in the same bits as without any weight
    import torch
    rng = np.random.default_rng(4)
    x, x64 = rounded(rng.standard_normal((2, 3, 9, 64)) * 3, torch.bfloat16)
    w, w64 = rounded(1 + 0.2 * rng.standard_normal(64), torch.bfloat16)
    f, pos = _freq(64), np.broadcast_to(np.arange(9), (2, 9))
    both = dd.dd_qk_norm_rope(x, x, q_weight=w if which == "queries" else None, k_weight=w if which == "keys" else None, inv_freq=dev(f))
    normed, plain = both if which == "queries" else both[::-1]
    assert torch.equal(plain, dd.dd_qk_norm_rope(x, inv_freq=dev(f))[0])
    assert_rows(host(normed), paged.norm_rope(x64, w64, float(np.float32(1e-6)), f, pos, False), 2.0 ** -8, ROW_FAST)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    import torch
    t, half_step, row = _types(dtype)
    rng = np.random.default_rng(1)
    pos = np.array([[0, -1, -70000, 2**24 + 1, 2**31 - 1, -2**31, 131071]])
    Q, q64 = rounded(rng.standard_normal((1, 2, 7, 128)), t)
    f = _freq(128, 500000.0)
    Qo, none = dd.dd_qk_norm_rope(Q, inv_freq=dev(f), positions=ints(pos))
    assert none is None
    assert_rows(host(Qo), paged.norm_rope(q64, None, 0, f, pos, False), half_step, row)


def test_many_tokens_many_heads_and_default_positions():
    # enough tokens that a workgroup goes through all heads, the last workgroup ragged; and layouts of the input against each other
    a = _check(1, 6, 2, 515, 64, "bf16", 64, True, False, positions=False)
    b = _check(1, 6, 2, 515, 64, "bf16", 64, True, False, positions=False, fused=False)
    assert np.array_equal(host(a[2]), host(b[2])) and np.array_equal(host(a[3]), host(b[3]))


def test_one_group_of_heads_for_each_workgroup_count():
    # rows of one token give the same whatever else is in the call: 1 token (a head per workgroup) and 70000 (all heads in one)
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    Q = torch.randn((1, 3, 70001, 64), generator=g, device="cuda").bfloat16()
    w = torch.ones(64, device="cuda").bfloat16()
    f = dev(_freq(64))
    whole, _ = dd.dd_qk_norm_rope(Q, q_weight=w, inv_freq=f)
    for i in (0, 31, 32, 69999, 70000):
        one, _ = dd.dd_qk_norm_rope(Q[:, :, i:i + 1], q_weight=w, inv_freq=f, positions=ints([[i]]))
        assert torch.equal(one, whole[:, :, i:i + 1])


def test_in_place_and_given_outputs():
    import torch
    rng = np.random.default_rng(2)
    Q, K = dev(rng.standard_normal((2, 4, 9, 64)), torch.float32), dev(rng.standard_normal((2, 2, 9, 64)), torch.float32)
    f = dev(_freq(64))
    want = dd.dd_qk_norm_rope(Q, K, inv_freq=f)
    Qo = torch.full_like(Q, float("nan"))
    got = dd.dd_qk_norm_rope(Q, K, inv_freq=f, Qo=Qo)
    assert got[0].data_ptr() == Qo.data_ptr() and torch.equal(Qo, want[0])
    dd.dd_qk_norm_rope(Q, K, inv_freq=f, Qo=Q, Ko=K)
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1])


def test_strides_zero_and_overlapping_rows():
    import torch
    rng = np.random.default_rng(3)
    base = dev(rng.standard_normal(64 * 40), torch.float32)
    Q = base.as_strided((2, 3, 5, 64), (0, 64, 128, 1))                       # a broadcast batch, rows that share elements
    got, _ = dd.dd_qk_norm_rope(Q, inv_freq=dev(_freq(64)))
    want, _ = dd.dd_qk_norm_rope(Q.contiguous(), inv_freq=dev(_freq(64)))
    assert torch.equal(got, want)


def test_rows_of_zeros_infinities_and_nan_stay_in_their_rows():
    import torch
    x = torch.randn((1, 1, 64, 128), device="cuda")
    x[0, 0, 3] = 0
    x[0, 0, 7, 5] = float("nan")
    x[0, 0, 11, 5] = float("inf")
    w = torch.ones(128, device="cuda")
    got, _ = dd.dd_qk_norm_rope(x, q_weight=w, inv_freq=dev(_freq(128)))
    assert not got[0, 0, 3].any() and got[0, 0, 7].isnan().all()
    clean = torch.ones(64, dtype=torch.bool, device="cuda")
    clean[[7, 11]] = False
    assert got[0, 0][clean].isfinite().all()


def test_no_tokens():
    import torch
    Qo, Ko = dd.dd_qk_norm_rope(torch.empty((2, 4, 0, 64), device="cuda"), torch.empty((2, 2, 0, 64), device="cuda"))
    assert Qo.shape == (2, 4, 0, 64) and Ko.shape == (2, 2, 0, 64)
