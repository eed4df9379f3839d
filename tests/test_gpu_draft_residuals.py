"""Draws of dd_verify_draft from what is left of the verifier's probabilities where that hangs on tokens that are almost as likely with the
drafter: the sums that say which of the two is the larger have to be good to fp64 there.  Against the fp64 oracle, wherever the mark is further
than NEAR from a border (test_gpu_verify_draft.py has its derivation), with marks 2e-11 to 1e-3 of the whole away from borders."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import draft
from _paged import dev, ints, rounded
from test_gpu_verify_draft import NEAR

pytestmark = pytest.mark.gpu


def _turned_down(v, d, dtype, seed, temperature=None, reach=1e-3, first=0):
    """One draft a row, of a token that the drafter likes better, by as much as it can be, which a random number of almost 1 turns down; the
    draw's number `reach` of the whole and less from a border at token `first` or behind."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(seed)
    (lv, v64), (ld, d64) = rounded(v, t), rounded(d, t)
    B, _, V = v.shape
    x, u = np.zeros((B, 1), np.int32), np.full((B, 2), 1 - 2.0 ** -24)
    for b in range(B):
        T = 1.0 if temperature is None else temperature[b]
        p, q = draft.probabilities(v64[b, 0], T), draft.probabilities(d64[b, 0], T)
        x[b, 0] = np.argmax(np.where(q > 0, q / np.maximum(p, 1e-300), 0))
        w = np.maximum(p - q, 0)
        c = np.cumsum(w)
        at = rng.choice(first + np.flatnonzero(w[first:]))
        off = np.exp(rng.uniform(np.log(2 * NEAR), np.log(max(reach * c[-1], 4 * NEAR)))) * rng.choice([-1, 1])
        u[b, 1] = min(max((c[at] + off) / c[-1], 2.0 ** -30), 1 - 2.0 ** -24)
    u = u.astype(np.float32)
    T = None if temperature is None else np.asarray(temperature, np.float32)
    args = dict(logits_v=lv, logits_d=ld, tokens=ints(x), uniforms=dev(u), temperature=None if T is None else dev(T))
    want = dict(logits_v=v64, logits_d=d64, tokens=x, uniforms=u.astype(np.float64), temperature=None if T is None else T.astype(np.float64), bonus=False)
    return args, want


def _check(args, want):
    tokens, accepted, _ = (t.cpu().numpy() for t in dd.dd_verify_draft(**args))
    w_tokens, w_accepted, _, margin = draft.verify_draft(**want)
    sure = margin > NEAR
    assert sure.sum() >= 2 and (w_accepted[sure] == 0).mean() >= 0.5       # (borders may be as close together as that)
    assert np.array_equal(accepted[sure], w_accepted[sure])
    wrong = sure & (tokens != w_tokens).any(1)
    assert not wrong.any(), f"{wrong.sum()} of {sure.sum()} rows: {tokens[wrong][:4].tolist()} for {w_tokens[wrong][:4].tolist()}"


@pytest.mark.parametrize("B,V", [(200, 1024), (16, 32000), (3, 152064)])
@pytest.mark.parametrize("noise", [1e-2, 1e-4, 1e-5, 1e-6])
def test_drafters_that_nearly_agree(B, V, noise):
    rng = np.random.default_rng(V + int(1 / noise))
    v = 2.0 * rng.standard_normal((B, 1, V))
    _check(*_turned_down(v, v + noise * rng.standard_normal(v.shape), "f32", seed=B))


@pytest.mark.parametrize("noise", [1e-3, 1e-5])
def test_drafters_that_nearly_agree_at_other_temperatures(noise):
    rng = np.random.default_rng(7)
    v = 2.0 * rng.standard_normal((60, 1, 4096))
    _check(*_turned_down(v, v + noise * rng.standard_normal(v.shape), "f32", seed=1, temperature=np.tile([0.25, 0.7, 1.5], 20)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V", [(200, 1024), (8, 64000)])
def test_logits_that_are_the_same_but_for_a_few(dtype, B, V):
    # every other token is as likely with either but for the quotient of the two sums, 1 and some 1e-6
    rng = np.random.default_rng(V)
    v = 2.0 * rng.standard_normal((B, 1, V)).astype(np.float32)
    d = v.copy()
    for b in range(B):
        some = rng.choice(np.flatnonzero(v[b, 0] < -3), 6, replace=False)
        d[b, 0, some] -= np.array([1, -1, 1, -1, 1, -1]) * (0.25 if dtype == "bf16" else 1e-2)
    _check(*_turned_down(v, d, dtype, seed=2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("apart", [0.0, 1e-7, 1e-6])
def test_one_token_that_both_think_as_likely(dtype, apart):
    # half of the probability on a token in front, to some 1e-7 the same with either, behind it tokens that the drafter likes better: what
    # comes next begins at a border of next to nothing
    B, V = 600, 1024
    rng = np.random.default_rng(int(apart * 1e8))
    v, d = rng.standard_normal((B, 1, V)), rng.standard_normal((B, 1, V))
    v[..., :256] -= 6
    v[..., 7] = d[..., 7] = 0
    if dtype == "bf16":
        import torch
        v, d = (torch.from_numpy(a).bfloat16().double().numpy() for a in (v, d))
    else:
        v, d = v.astype(np.float32).astype(np.float64), d.astype(np.float32).astype(np.float64)
    # token 7: the others' sum, as far as logits can be set
    rest = lambda a: np.log(np.exp(a).sum(-1) - np.exp(a[..., 7]))
    v[..., 7], d[..., 7] = rest(v), rest(d) + apart
    _check(*_turned_down(v, d, dtype, seed=3, reach=1e-6, first=256))


def test_a_call_repeats_itself():
    import torch
    rng = np.random.default_rng(5)
    v = 2.0 * rng.standard_normal((40, 1, 8192))
    args, _ = _turned_down(v, v + 1e-5 * rng.standard_normal(v.shape), "f32", seed=4)
    want = dd.dd_verify_draft(**args)
    assert all(all(torch.equal(a, b) for a, b in zip(want, dd.dd_verify_draft(**args))) for _ in range(5))
