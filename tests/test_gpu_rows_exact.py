"""How exact the rotation of fp32 rows is: to its last bits, as fp32 rows are taken for that."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from _paged import dev, host, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("far", [200, 200000, 2**31 - 1])
def test_fp32_rotation(far, interleaved):
    # Sine and cosine are off by at most one step, 2^-24 (they are below 1), and their correction by what the fp32 angle leaves out rounds
    # once more: 1.5 x 2^-24 each, for a pair of length r sqrt 2 x 1.5 x 2^-24 r < 2.13; two products of lengths that add to r at most,
    # 2^-24 r; their sum, 2^-24 r: 4.13 x 2^-24 r in all, and second-order terms far below the rest of 4.25.
    import torch
    rng = np.random.default_rng(far % 1000 + interleaved)
    d, n = 128, 4096
    x = rng.standard_normal((1, 2, n, d)).astype(np.float32)
    f = (500000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    pos = rng.integers(-far, far, (1, n))
    got, _ = dd.dd_qk_norm_rope(dev(x), inv_freq=dev(f), positions=ints(pos), interleaved=interleaved)
    a = pos[0].astype(np.longdouble)[:, None] * f.astype(np.longdouble)
    c, s = np.cos(a).astype(np.float64), np.sin(a).astype(np.float64)
    pair = (lambda y: (y[..., 0::2], y[..., 1::2])) if interleaved else (lambda y: (y[..., :d // 2], y[..., d // 2:]))
    (u, v), (gu, gv) = pair(x.astype(np.float64)), pair(host(got))
    r = np.hypot(u, v)
    worst = max((np.abs(gu - (u * c - v * s)) / r).max(), (np.abs(gv - (v * c + u * s)) / r).max())
    assert worst <= 4.25 * 2.0 ** -24, f"{worst * 2.0 ** 24:.2f} x 2^-24"
