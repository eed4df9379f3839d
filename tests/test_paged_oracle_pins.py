"""Pins of the paged oracle (oracle/paged.py): closed forms, invariants, torch's conversions.  CPU only."""
import numpy as np
import pytest

import oracle
from oracle import paged


def test_e4m3_is_the_decode_table_and_torch():
    import torch
    codes = np.arange(256, dtype=np.uint8)
    finite = (codes & 0x7f) != 0x7f
    values = np.array([oracle.decode_e4m3(int(c)) for c in codes])
    assert np.array_equal(paged.e4m3(values[finite]), values[finite])
    x = np.concatenate([np.random.default_rng(0).standard_normal(4000) * s for s in (1e-3, 0.02, 1, 60)]).clip(-448, 448).astype(np.float32)
    pos = np.sort(values[finite & (codes < 128)])
    mid = ((pos[1:] + pos[:-1]) / 2).astype(np.float32)                    # ties
    x = np.concatenate([x, mid, -mid])
    assert np.array_equal(paged.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_scale_is_least():
    for a in (1e-3, 0.1, 1.75, 1.7500001, 3.5, 7.0, 447.9, 448.0, 448.1, 1e4):
        s = paged.scale_for(a)
        assert a <= 448 * s and a > 448 * s / 2
    assert paged.scale_for(0.0) == 2.0 ** -126


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation(interleaved):
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 64))
    f = 10000.0 ** (-np.arange(16) / 16)                                     # 32 of 64 dims turn
    at = lambda v, p: paged.norm_rope_row(v, None, 0, f, p, interleaved)
    assert np.array_equal(at(x, 0), x)                                       # position 0
    assert np.allclose(np.linalg.norm(at(x, 77)), np.linalg.norm(x))
    assert np.allclose(at(x, 19) @ at(y, 12), at(x, 107) @ at(y, 100))       # only the distance counts
    assert np.array_equal(at(x, 9)[32:], x[32:])                             # the rest stays
    e = np.zeros(64)
    e[0] = 1                                                                 # the first pair turns by the position itself
    r = at(e, 1)
    assert np.isclose(r[0], np.cos(1)) and np.isclose(r[1 if interleaved else 16], np.sin(1)) and np.count_nonzero(r) == 2


def test_norm():
    x = np.full(64, -3.0)
    assert np.allclose(paged.norm_rope_row(x, np.full(64, 2.0), 1e-12, None, 5, False), -2.0)
    x = np.random.default_rng(2).standard_normal(128)
    assert np.allclose(paged.norm_rope_row(x, np.ones(128), 1e-9, None, 0, False), paged.norm_rope_row(100 * x, np.ones(128), 1e-5, None, 0, False), rtol=1e-8)


def _dense(cache, table, b, n, values):
    c = cache.swapaxes(-1, -2) if values else cache
    return np.concatenate([c[p] for p in table[b]], axis=1)[:, :n]           # [Hkv, n, d]


def test_append_places_rows_and_attention_reads_them():
    rng = np.random.default_rng(3)
    B, Hkv, P, d, n = 2, 2, 16, 64, 37
    table = rng.permutation(9)[:8].reshape(B, 4)
    Kc, Vc = rng.standard_normal((9, Hkv, P, d)), rng.standard_normal((9, Hkv, d, P))
    K, V = rng.standard_normal((2, B, Hkv, n, d))
    Kn, Vn, _, _, _ = paged.paged_append(Kc, Vc, None, None, K, V, table, [0, 11])
    for b, s in enumerate((0, 11)):
        assert np.array_equal(_dense(Kn, table, b, s + n, False)[:, s:], K[b]) and np.array_equal(_dense(Vn, table, b, s + n, True)[:, s:], V[b])
        assert np.array_equal(_dense(Kn, table, b, s, False), _dense(Kc, table, b, s, False))
    Q = rng.standard_normal((B, 4, 3, d))
    O, _ = paged.paged_attention(Q, Kn, Vn, None, None, table, [n, 0])
    want = oracle.block_attention_cached(Q[:1], K[:1].copy(), V[:1].copy(), 0, oracle.F64, oracle.F64)     # the dense oracle on the same rows
    assert np.allclose(O[0], want[0], atol=1e-12) and not O[1].any()


def test_append_scales():
    rng = np.random.default_rng(4)
    P, d = 16, 64
    zeros = np.zeros((1, 1, P, d)), np.zeros((1, 1, d, P))
    K = rng.standard_normal((1, 1, P, d))
    Kc, Vc, ks, vs, _ = paged.paged_append(*zeros, np.ones((1, 1)), np.ones((1, 1)), K, 8 * K, [[0]], [0])
    assert ks[0, 0] == paged.scale_for(np.abs(K).max()) and vs[0, 0] == 8 * ks[0, 0]
    assert np.abs(Kc * ks[0, 0] - K).max() <= np.abs(K).max() / 16
    # a larger row is added: its page grows by powers of two, and what was there keeps its values (but for subnormal codes)
    big = 100 * K[:, :, :1]
    K2, _, ks2, _, _ = paged.paged_append(Kc, Vc, ks, vs, big, big, [[0]], [10])
    assert ks2[0, 0] == paged.scale_for(np.abs(big).max()) > ks[0, 0]
    held = np.abs(K2[0, 0, :10]) > 2.0 ** -6                                 # (2^-6 itself may have been rounded up from a subnormal number)
    assert held.any() and np.array_equal((K2 * ks2)[0, 0, :10][held], (Kc * ks)[0, 0, :10][held])
    # a smaller one leaves the scale; a page that keeps nothing takes the scale of its rows
    small = 1e-3 * K[:, :, :1]
    assert paged.paged_append(Kc, Vc, ks, vs, small, small, [[0]], [10])[2] == ks
    assert paged.paged_append(Kc, Vc, ks, vs, small, small, [[0]], [0])[2] == paged.scale_for(np.abs(small).max())
    assert paged.paged_append(Kc, Vc, ks, vs, small, small, [[0]], [0], kv_lens=[2])[2] == ks


def test_positions_and_pages_out_of_range_are_skipped():
    rng = np.random.default_rng(5)
    Kc, Vc = rng.standard_normal((2, 1, 16, 64)), rng.standard_normal((2, 1, 64, 16))
    K = rng.standard_normal((1, 1, 40, 64))
    got = paged.paged_append(Kc, Vc, None, None, K, K, [[7, 1]], [-3])
    assert np.array_equal(got[0][0], Kc[0]) and np.array_equal(got[0][1, 0], K[0, 0, 19:35])
    O, _ = paged.paged_attention(rng.standard_normal((1, 1, 1, 64)), Kc, Vc, None, None, [[7, -1]], [32])
    assert not O.any()
