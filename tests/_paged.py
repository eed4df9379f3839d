"""Inputs and comparisons shared by the tests of head norms with rotation and of the paged cache."""
import numpy as np

import oracle

E4M3 = np.array([oracle.decode_e4m3(c) for c in range(256)])


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).to("cuda:0")
    return t if dtype is None else t.to(dtype)


def ints(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to("cuda:0")


def host(t):
    """the numbers that a device tensor holds, fp64"""
    import torch
    return t.view(torch.uint8).cpu().numpy().astype(np.int64) if t.dtype == torch.uint8 else t.detach().cpu().to(torch.float64).numpy()


def rounded(x, dtype):
    """x as the device holds it in `dtype`: (device tensor, its numbers)"""
    t = dev(np.asarray(x, np.float32), dtype)
    return t, host(t)


def fp8_cache(rng, shape, lo=-8, hi=-4, poison=False):
    """random e4m3 pages and power-of-two scales: (codes on the device, numbers, scales on the device, scales)"""
    import torch
    codes = rng.integers(0, 256, shape, dtype=np.uint8)
    codes[(codes & 0x7f) == 0x7f] = 0x38
    scale = (2.0 ** rng.integers(lo, hi, shape[:2])).astype(np.float32)
    return dev(codes).view(torch.float8_e4m3fn), E4M3[codes], dev(scale), scale.astype(np.float64)


def codes_of(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


# What fp32 arithmetic may add before the rounding of a result, relative to the largest magnitude of a row.  A normed element is off by
# at most 10 (the sum of squares, halved by the root) + 5 (root, reciprocal, products) = 15 steps of 2^-24 relative; a rotation adds
# |u| + |v| <= 2 max times 3 (products and sum) + 3 (fraction of a revolution in fp32) + 2 (sinpi) steps, and the 15 of both of its
# members: 2 x (15 + 8) = 46 < 64 steps, 2^-18.  The hardware's sine and cosine, used for bf16 and e4m3 results, are off by up to
# 2^-19: 2 x 2^-19 more, under 2^-17 in all.
ROW_F32, ROW_FAST = 2.0 ** -18, 2.0 ** -17


def assert_rows(got, want, half_step, row_error, what=""):
    """|got - want| <= half a step of the result's type, relative, + the arithmetic's share of the row's largest magnitude"""
    top = np.abs(want).max(-1, keepdims=True)
    tol = half_step * np.abs(want) + row_error * (1 + half_step) * top
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} elements off, worst {np.abs(got - want)[bad].max():.3e} at {np.argwhere(bad)[:3].tolist()}"


def attention_tolerance(O, A):
    """Weights are rounded to bf16 (2^-8 of each at most: 2^-8 A), the result again (2^-8 |O|); scores are fp32 sums of up to 128
    products whose magnitudes add to some 30 at most here, times log2 e: 140 steps of 2^-24 x 45 < 2^-11 of each weight, in O and in
    its divisor."""
    return (2.0 ** -8 + 2 * 2.0 ** -11) * A + 2.0 ** -8 * np.abs(O) + 1e-30
