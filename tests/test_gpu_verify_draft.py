"""GPU parity of dd_verify_draft against the fp64 oracle.  Tokens and counts are equal wherever the oracle's closest decision is further from
its border than fp64 sums and exponentials good to 1.1e-12 can move it: a probability is a quotient of two such sums, a decision compares
two of them, a draw sums differences of two - at most 8 errors, next to weights that add to at most 1.
Chances are quotients of fp32 sums: an exponent's two roundings and its factor's, 2^-24 each of 40 at most (what is below adds less than
2^-40 of a sum per token), times ln 2, the exponential's own 2^-23 and three additions of 2^-24 are 5.5e-6 of a sum, two of which meet."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import draft
from paper_2604_05250_amd.step import capture_step
from _paged import dev, host, ints, rounded
from test_gpu_guard_bands import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu

NEAR = 1e-11
CHANCE = 2 * (3 * 40 * np.log(2) + 2 + 3) * 2.0 ** -24 + 2.0 ** -24


def _case(B, n, V, dtype="bf16", seed=0, sure=False, temperature=None, n_draft=None, bonus=True, sigma=3.0, holes=0.0):
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(seed)
    rows = n + bool(bonus)
    d = sigma * rng.standard_normal((B, rows, V))
    v = d + sigma / 3 * rng.standard_normal((B, rows, V))
    if holes:                                                # tokens that a filter took out of either
        v[rng.random(v.shape) < holes] = -np.inf
        d[rng.random(d.shape) < holes] = -np.inf
        v[..., 0], d[..., 1] = 0.0, 0.0
    lv, v64 = rounded(v, t)
    ld, d64 = rounded(d[:, :n], t)
    temps = np.ones(B) if temperature is None else np.asarray(temperature, np.float32).astype(np.float64)
    x = np.zeros((B, n), np.int32)
    for b in range(B):
        for i in range(n):
            q = draft.probabilities(d64[b, i], temps[b])
            x[b, i] = rng.choice(V, p=q / q.sum())
    u = rng.random((B, n + 1)).astype(np.float32)
    u[u >= 1] = 0.5
    args = dict(logits_v=lv, logits_d=None if sure else ld, tokens=ints(x), uniforms=dev(u),
                temperature=None if temperature is None else dev(np.asarray(temperature, np.float32)), n_draft=None if n_draft is None else ints(n_draft))
    want = dict(logits_v=v64, logits_d=None if sure else d64, tokens=x, uniforms=u.astype(np.float64),
                temperature=None if temperature is None else temps, n_draft=n_draft, bonus=bonus)
    return args, want


def _compare(got, want, strict=True):
    tokens, accepted, chances = (t.cpu().numpy() for t in got)
    w_tokens, w_accepted, w_chances, margin = draft.verify_draft(**want)
    sure = margin > NEAR
    assert sure.mean() >= 0.5 or not strict
    assert np.array_equal(accepted[sure], w_accepted[sure]), (accepted, w_accepted)
    assert np.array_equal(tokens[sure], w_tokens[sure]), np.argwhere(tokens != w_tokens)
    assert (np.abs(chances - w_chances) <= CHANCE * w_chances + 2.0 ** -149).all()


def _check(*a, **kw):
    args, want = _case(*a, **kw)
    got = dd.dd_verify_draft(**args)
    _compare(got, want)
    return args, want, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,V", [(1, 1, 8), (2, 3, 24), (3, 1, 4096), (5, 4, 1000), (1, 8, 32000), (9, 2, 12344), (2, 2, 126464), (70, 1, 2056), (1, 40, 520)])
def test_parity(dtype, B, n, V):
    _check(B, n, V, dtype=dtype, seed=V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sure", [False, True])
@pytest.mark.parametrize("bonus", [False, True])
def test_ragged_drafts_and_temperatures(dtype, sure, bonus):
    B, n = 12, 5
    _check(B, n, 3000, dtype=dtype, sure=sure, bonus=bonus, temperature=[0.0, 0.3, 1.0, 2.5, 0.0, 0.7, 1e-7, 1.3, 40.0, 0.05, 1.0, 0.0],
           n_draft=[0, 1, 2, 3, 4, 5, 5, 9, -3, 5, 5, 0], seed=sure + 2 * bonus)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_impossible_tokens(dtype):
    _check(20, 3, 400, dtype=dtype, holes=0.6, seed=5)
    _check(20, 3, 400, dtype=dtype, holes=0.6, seed=6, sure=True, temperature=[0.0, 1.0] * 10)


def test_no_draft_at_all_draws_from_the_verifier():
    import torch
    args, want = _case(7, 0, 5000, seed=3)
    got = dd.dd_verify_draft(**args)
    assert got[0].shape == (7, 1) and got[2].shape == (7, 0)
    _compare(got, want)
    assert torch.equal(dd.dd_verify_draft(args["logits_v"], None, args["tokens"], args["uniforms"])[0], got[0])


def test_every_position_on_its_own():
    # the marginals of a masked diffusion model: one draft a sequence, no row behind it
    B, n, V = 4, 32, 1024
    args, want = _case(B, n, V, bonus=False, seed=8)
    flat = lambda t, *s: t.reshape(B * n, *s)
    u = np.random.default_rng(1).random((B * n, 2)).astype(np.float32)
    got = dd.dd_verify_draft(flat(args["logits_v"], 1, V), flat(args["logits_d"], 1, V), flat(args["tokens"], 1), dev(u))
    _compare(got, dict(logits_v=flat(want["logits_v"], 1, V), logits_d=flat(want["logits_d"], 1, V), tokens=flat(want["tokens"], 1),
                       uniforms=u.astype(np.float64), bonus=False))
    kept = got[1].cpu().numpy() == 1
    assert kept.any() and (~kept).any() and (got[0].cpu().numpy()[kept, 1] == -1).all() and (got[0].cpu().numpy()[~kept, 0] >= 0).all()


def test_equal_rows_keep_every_draft():
    import torch
    args, _ = _case(6, 4, 2048, seed=1)
    args["logits_d"] = args["logits_v"][:, :4].contiguous()
    args["uniforms"] = torch.full((6, 5), 1 - 2.0 ** -24, device="cuda")
    tokens, accepted, chances = dd.dd_verify_draft(**args)
    assert bool((accepted == 4).all()) and torch.equal(tokens[:, :4], args["tokens"]) and bool((chances == 1).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_marks_next_to_borders(dtype):
    # the random numbers stand right next to a draft's chance and to borders between tokens: 2^-24 beside them, where fp32 sums would miss
    B, n, V = 32, 1, 8192
    args, want = _case(B, n, V, dtype=dtype, seed=11, sigma=1.0)
    chance = draft.verify_draft(**want)[2][:, 0]
    u = want["uniforms"].copy()
    for b in range(B):
        u[b, 0] = np.floor(chance[b] * 2 ** 24) / 2 ** 24 if b % 2 else np.ceil(chance[b] * 2 ** 24) / 2 ** 24
        u[b, 0] = min(u[b, 0], 1 - 2.0 ** -24)
        p = draft.probabilities(want["logits_v"][b, 0], 1.0)
        w = np.maximum(p - draft.probabilities(want["logits_d"][b, 0], 1.0), 0) if not u[b, 0] < chance[b] else draft.probabilities(want["logits_v"][b, 1], 1.0)
        c = np.cumsum(w) / w.sum()
        mark = c[(37 * b) % V]
        u[b, 1] = min((np.floor if b % 3 else np.ceil)(mark * 2 ** 24) / 2 ** 24, 1 - 2.0 ** -24)
    args["uniforms"], want["uniforms"] = dev(u.astype(np.float32)), u
    _compare(dd.dd_verify_draft(**args), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_from_zero_and_far_apart(dtype):
    # logits around +-1e4 and a spread of 1e4: references, powers that are none
    args, want = _case(8, 2, 640, dtype=dtype, seed=2, sigma=3000.0)
    shift = np.array([1e4, -1e4, 0, 1e4, -1e4, 1, 2, 3])[:, None, None]
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    args["logits_v"], want["logits_v"] = rounded(want["logits_v"] + shift, t)
    args["logits_d"], want["logits_d"] = rounded(want["logits_d"] - shift, t)
    _compare(dd.dd_verify_draft(**args), want)


def test_values_outside_the_contract_stay_inside_the_tensors():
    import torch
    g = Guarded()
    B, n, V = 6, 3, 264
    lv = g.empty((B, n + 1, V), torch.float32)
    lv.normal_()
    lv[0] = float("nan")
    lv[1] = float("-inf")
    lv[2, 1, 5] = float("inf")
    lv[3] = 3e38
    ld = torch.randn((B, n, V), device="cuda")
    tokens = ints([[-1, 2, 3], [2 ** 31 - 1, 0, 0], [-2 ** 31, 1, 1], [V, V, V], [5, V, 5], [1, 2, 3]])
    u = dev(np.array([[0, 0, 0, np.nan], [0, 0, 0, 0.5], [np.nan] * 4, [2, 2, 2, 2], [-1, -1, -1, -1], [0.1, 0.2, np.inf, np.inf]], np.float32))
    out = g.empty((B, n + 1), torch.int32), g.empty((B,), torch.int32), g.empty((B, n), torch.float32)
    for temperature in (None, dev(np.array([1, np.nan, -1, np.inf, 0, 1e-3], np.float32))):
        for d in (ld, None):
            with dd.fixed_workspace(guarded_workspace(g, dd.dd_verify_draft_workspace_bytes(B, n, 1, V, d is not None, dd.F32))):
                dd.dd_verify_draft(lv, d, tokens, u, temperature=temperature, out_tokens=out[0], out_accepted=out[1], out_chances=out[2])
            g.check("odd values")
            a, x = out[1].tolist(), out[0].tolist()
            for b in range(B):
                assert 0 <= a[b] <= n and x[b][:a[b]] == tokens[b].tolist()[:a[b]] and -1 <= x[b][a[b]] < V and x[b][a[b] + 1:] == [-1] * (n - a[b])
            assert x[1][0] == (-1 if temperature is None else 0) and a[1] == 0       # no probability anywhere; a temperature of NaN is 0


@pytest.mark.parametrize("dtype,V", [("bf16", 8), ("bf16", 126464), ("f32", 1236)])
def test_nothing_else_is_written(dtype, V):
    import torch
    args, want = _case(3, 2, V, dtype=dtype, seed=4, n_draft=[2, 1, 0])
    kept = {k: v.clone() for k, v in args.items() if v is not None}
    g = Guarded()
    out = g.empty((3, 3), torch.int32), g.empty((3,), torch.int32), g.empty((3, 2), torch.float32)
    need = dd.dd_verify_draft_workspace_bytes(3, 2, 1, V, 1, dd.BF16 if dtype == "bf16" else dd.F32)
    with dd.fixed_workspace(g.empty((need,), torch.uint8)):
        got = dd.dd_verify_draft(**args, out_tokens=out[0], out_accepted=out[1], out_chances=out[2])
    g.check(f"{dtype} V {V}")
    assert [t.data_ptr() for t in got] == [t.data_ptr() for t in out]
    assert all(torch.equal(args[k], v) for k, v in kept.items())
    _compare(got, want)


def test_rows_behind_the_last_are_not_read():
    import torch
    args, want = _case(4, 3, 1000, seed=9, n_draft=[0, 1, 2, 3])
    for b in range(4):
        args["logits_v"][b, b + 1:] = float("nan")
        args["logits_d"][b, b:] = float("nan")
        args["tokens"][b, b:] = -2 ** 31
    _compare(dd.dd_verify_draft(**args), want)


def test_graph_replays_match_eager_calls():
    import torch
    args, _ = _case(3, 4, 30000, seed=12, temperature=[0.0, 0.8, 1.0])
    out = torch.zeros((3, 5), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((3, 4), device="cuda")

    def step():
        dd.dd_verify_draft(**args, out_tokens=out[0], out_accepted=out[1], out_chances=out[2])

    graph = capture_step(step)
    for rep in range(5):
        args["uniforms"].copy_(torch.rand((3, 5), generator=torch.Generator().manual_seed(rep)))
        args["logits_v"].copy_(args["logits_v"].roll(1, 0))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in out]
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), f"replay {rep}"


def test_streams_side_by_side():
    import torch
    cases = [_case(2, 3, 20000, seed=k)[0] for k in range(3)]
    want = [dd.dd_verify_draft(**c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[] for _ in cases]
    for _ in range(5):
        for c, s, to in zip(cases, streams, got):
            with torch.cuda.stream(s):
                to.append(dd.dd_verify_draft(**c))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for w, gs in zip(want, got) for g in gs for a, b in zip(w, g))


def test_offsets_past_32_bits():
    # rows of 2^27 fp32 logits, nine of them: a spike that stands, one that falls, and flat rows, where token floor(u V) is drawn
    import torch
    V, B, n = 1 << 27, 3, 2
    lv, ld = torch.zeros((B, n + 1, V), device="cuda"), torch.zeros((B, n, V), device="cuda")
    x = np.array([[V - 1, 5], [V - 2, 7], [V - 3, 9]], np.int32)
    for b in range(B):
        ld[b, 0, int(x[b, 0])] = lv[b, 0, int(x[b, 0])] = 60.0           # as likely with either: stands
    lv[1, 1, V - 9], ld[1, 1, 7] = 60.0, 60.0                            # the drafter's favourite has no chance
    k = [(1 << 24) - 1, 77, (1 << 24) - 5]
    u = np.array([[0.5, 0.5, k[0] / 2 ** 24], [0.5, 0.5, k[1] / 2 ** 24], [0.5, 0.5, k[2] / 2 ** 24]], np.float32)
    out, accepted, _ = dd.dd_verify_draft(lv, ld, ints(x), dev(u))
    assert accepted.tolist() == [2, 1, 2]
    assert out.tolist() == [[V - 1, 5, 8 * k[0]], [V - 2, V - 9, -1], [V - 3, 9, 8 * k[2]]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("u", [0.0, 1 - 2.0 ** -24])
def test_random_numbers_at_their_ends(dtype, u):
    # 0 keeps every draft that is possible and draws the first token that is, the largest number the last one
    args, want = _case(16, 3, 320, dtype=dtype, holes=0.5, seed=21)
    want["uniforms"] = np.full((16, 4), u)
    args["uniforms"] = dev(want["uniforms"].astype(np.float32))
    args["tokens"][::2] = ints(np.random.default_rng(0).integers(0, 320, (8, 3)))
    want["tokens"] = args["tokens"].cpu().numpy()
    tokens, accepted, _, margin = draft.verify_draft(**want)
    got = dd.dd_verify_draft(**args)
    sure = (margin > NEAR) | (u == 0)                        # (0 is no further from the first border than that token's own weight)
    assert sure.any() and np.array_equal(got[1].cpu().numpy()[sure], accepted[sure]) and np.array_equal(got[0].cpu().numpy()[sure], tokens[sure])


def test_temperatures_far_out():
    # very hot: all tokens that are possible alike; very cold: the largest logit, from 1e-6 down by rule
    temps = [1e30, 3e38, 1e6, 2e-6, 1e-4, 1e-6, 1e-38, 0.0]
    args, want = _case(8, 3, 512, temperature=[1.0] * 8, holes=0.3, seed=13)
    args["temperature"], want["temperature"] = dev(np.array(temps, np.float32)), np.array(temps, np.float32).astype(np.float64)
    _compare(dd.dd_verify_draft(**args), want)


def test_many_sequences_and_the_same_memory_on_both_sides():
    import torch
    B, V = 5000, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    lv = torch.randn((B, 1, V), generator=g, device="cuda")
    tokens = torch.randint(0, V, (B, 1), generator=g, device="cuda").int()
    u = torch.rand((B, 2), generator=g, device="cuda")
    out, accepted, chances = dd.dd_verify_draft(lv, lv, tokens, u)
    assert bool((accepted == 1).all()) and torch.equal(out[:, :1], tokens) and bool((out[:, 1] == -1).all()) and bool((chances == 1).all())
    ld = torch.randn((B, 1, V), generator=g, device="cuda")
    _compare(dd.dd_verify_draft(lv, ld, tokens, u), dict(logits_v=host(lv), logits_d=host(ld), tokens=tokens.cpu().numpy(), uniforms=host(u), bonus=False))


def test_tokens_come_out_with_the_verifiers_probabilities():
    # drafts drawn from q, three hundred thousand of them: counts of the first token against p, chi squared with 15 degrees of freedom
    import torch
    B, V = 300000, 16
    g = torch.Generator(device="cuda").manual_seed(7)
    l = torch.randn((2, V), generator=g, device="cuda") * 1.5
    tokens = torch.multinomial(torch.softmax(l[1], 0), B, replacement=True, generator=g).int()[:, None]
    lv, ld = l[0].expand(B, 1, V).contiguous(), l[1].expand(B, 1, V).contiguous()
    for d in (ld, None):
        x = tokens if d is not None else torch.full_like(tokens, 3)
        out, accepted, _ = dd.dd_verify_draft(lv, d, x, torch.rand((B, 2), generator=g, device="cuda"))
        counts = torch.bincount(out[:, 0].long(), minlength=V).double()
        p = torch.softmax(l[0].double(), 0)
        chi2 = float(((counts - B * p) ** 2 / (B * p)).sum())
        assert chi2 < 60, chi2                               # (a chance of 2e-7)
