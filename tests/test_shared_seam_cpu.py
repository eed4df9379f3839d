"""That the comparison of test_gpu_shared_seam.py sees what it is there for: mistakes of one position at either end of a prefix or of a
sequence's own keys, planted into the oracle, fall outside its tolerance for every sequence that they concern."""
import numpy as np
import pytest

from test_gpu_shared_seam import SIZES, close, marked, wanted


@pytest.mark.parametrize("size", SIZES)
def test_a_position_more_or_less_is_seen(size):
    starts, H, Hkv, n, d, P, prefix_lens, lens = size
    n = min(n, 3)
    Q, K, V, ptable, table = marked(starts, H, Hkv, n, d, P, prefix_lens, lens)
    want = wanted(Q, K, V, ptable, prefix_lens, starts, table, lens)
    seen = lambda got: (~close(got, want)).any((1, 2, 3))
    assert not seen(want).any()
    assert seen(wanted(Q, K, V, ptable, [x - 1 for x in prefix_lens], starts, table, lens)).all()
    assert seen(wanted(Q, K, V, ptable, prefix_lens, starts, table, [x - 1 for x in lens])).all()
    # own positions that begin one behind their first
    K2, V2 = K.copy(), V.copy()
    for row in table:
        flat_k = np.concatenate([K[p] for p in row], 1)      # [Hkv, positions, d]
        flat_v = np.concatenate([V[p] for p in row], 2)
        flat_k, flat_v = np.roll(flat_k, -1, 1), np.roll(flat_v, -1, 2)
        for i, p in enumerate(row):
            K2[p], V2[p] = flat_k[:, i * P:(i + 1) * P], flat_v[:, :, i * P:(i + 1) * P]
    assert seen(wanted(Q, K2, V2, ptable, prefix_lens, starts, table, lens))[np.array(lens) % (P * table.shape[1]) != 0].all()
    # the prefix's last page in place of its first
    turned = [list(row[:-(-x // P)][::-1]) + list(row[-(-x // P):]) for row, x in zip(ptable, prefix_lens)]
    short = [x - 1 for x in prefix_lens]                     # (its last position is not there)
    assert seen(wanted(Q, K, V, turned, short, starts, table, lens)).all()
