"""Pins of the oracle of drafted tokens' verification: closed forms, and the property that the rule exists for - tokens come out with the
verifier's probabilities - by summing over a grid of the random numbers."""
import numpy as np
import pytest

from oracle import draft


def _logits(*p):
    return np.log(np.asarray(p, np.float64))


def test_a_draft_stands_with_probability_p_over_q():
    lv, ld = np.broadcast_to(_logits(0.1, 0.2, 0.7), (1, 2, 3)), np.broadcast_to(_logits(0.4, 0.4, 0.2), (1, 1, 3))
    for x, want in ((0, 0.25), (1, 0.5), (2, 1.0)):
        us = (np.arange(1000) + 0.5) / 1000
        kept = [draft.verify_draft(lv, ld, [[x]], [[u, 0.5]])[1][0] for u in us]
        assert abs(np.mean(kept) - want) < 1e-9
        assert abs(draft.verify_draft(lv, ld, [[x]], [[0.0, 0.5]])[2][0, 0] - want) < 1e-12


@pytest.mark.parametrize("sure", [False, True])
def test_tokens_come_out_with_the_verifiers_probabilities(sure):
    # the first token, over drafts x ~ q and a grid of (u_0, u_1): rationals whose borders the grid's middles never meet
    p, q = np.array([0.125, 0.25, 0.5, 0.125]), np.array([0.5, 0.25, 0.125, 0.125])
    lv, ld = np.broadcast_to(_logits(*p), (1, 2, 4)), np.broadcast_to(_logits(*q), (1, 1, 4))
    grid = (np.arange(64) + 0.5) / 64
    got = np.zeros(4)
    for x in range(4):
        for u0 in grid:
            for u1 in grid:
                out, a, _, _ = draft.verify_draft(lv, None if sure else ld, [[x]], [[u0, u1]])
                got[out[0, 0]] += q[x] / 64 ** 2
                assert a[0] == (out[0, 1] >= 0)
    # (where the drafter was sure, what is left are sevenths and thirds: a token's two borders are off by half a cell of u_1 each at most)
    assert np.abs(got - p).max() < (1e-9 if not sure else 1 / 64)


def test_draws_are_the_inverse_of_the_running_sum():
    w = np.array([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    assert [draft.draw(w, u)[0] for u in (0.0, 0.2499, 0.25, 0.5, 0.7499, 0.75, 0.999, 1.0, 7.0)] == [1, 1, 3, 3, 3, 4, 4, 4, 4]


def test_temperature_zero_takes_the_first_of_the_largest():
    lv = np.array([[[1.0, 3.0, 3.0, 2.0], [5.0, 5.0, 0.0, 0.0]]])
    for x, want in ((1, [1, 0]), (2, [1, -1]), (0, [1, -1])):
        out, a, c, _ = draft.verify_draft(lv, None, [[x]], [[0.999, 0.999]], temperature=[0.0])
        assert out[0].tolist() == want and a[0] == (x == 1) and c[0, 0] == (x == 1)


def test_lengths_and_rows_behind_the_drafts():
    rng = np.random.default_rng(0)
    lv, ld = rng.standard_normal((3, 4, 7)), np.full((3, 3, 7), -np.inf)
    ld[..., 0] = 0.0                                                        # a drafter that never draws what is drafted: q = 0
    out, a, c, _ = draft.verify_draft(lv, ld, np.full((3, 3), 5), np.full((3, 4), 0.5), n_draft=[0, 2, 9])
    assert a.tolist() == [0, 2, 3] and (c == [[0, 0, 0], [1, 1, 0], [1, 1, 1]]).all()
    assert (out[0, 1:] == -1).all() and out[1].tolist()[:2] == [5, 5] and out[1, 2] >= 0 and out[1, 3] == -1 and out[2, 3] >= 0
    assert (draft.verify_draft(lv[:, :3], ld, np.full((3, 3), 5), np.full((3, 4), 0.5), n_draft=[0, 2, 9], bonus=False)[0][[0, 1, 2], [0, 2, 3]] == -1).all()


def test_nothing_left_of_p_draws_from_p():
    lv = np.broadcast_to(_logits(0.5, 0.5), (1, 2, 2))
    out, a, _, _ = draft.verify_draft(lv, lv[:, :1], [[9]], [[0.5, 0.6]])   # no token of the vocabulary, and p == q
    assert a[0] == 0 and out[0].tolist() == [1, -1]
