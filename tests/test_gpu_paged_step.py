"""The calls around a paged cache as a serving loop makes them: prompts in, blocks drafted over them, the verifier's call on the same
rows; as a replayed graph, on several streams at once, inside guard bands."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import paged
from paper_2604_05250_amd.step import capture_step
from _paged import E4M3, ROW_FAST, assert_rows, attention_tolerance, codes_of, dev, host, ints, rounded
from test_gpu_guard_bands import Guarded, guarded_workspace

pytestmark = pytest.mark.gpu


class Served:
    """A batch of sequences on a paged cache, and its projections' outputs."""

    def __init__(self, B=3, H=8, Hkv=2, d=128, P=64, prompt=150, bl=16, steps=2, cache="fp8", seed=0):
        import torch
        rng = np.random.default_rng(seed)
        self.B, self.H, self.Hkv, self.d, self.bl, self.prompt = B, H, Hkv, d, bl, prompt
        per = -(-(prompt + steps * bl) // P)
        pages = B * per + 1
        self.table = ints(rng.permutation(pages)[:B * per].reshape(B, per))
        t = torch.uint8 if cache == "fp8" else torch.bfloat16
        self.Kc, self.Vc = torch.zeros((pages, Hkv, P, d), dtype=t, device="cuda"), torch.zeros((pages, Hkv, d, P), dtype=t, device="cuda")
        self.ks = self.vs = None
        if cache == "fp8":
            self.ks, self.vs = torch.ones((pages, Hkv), device="cuda"), torch.ones((pages, Hkv), device="cuda")
        self.freq = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
        self.f = dev(self.freq)
        self.qw, self.qw64 = rounded(1 + 0.2 * rng.standard_normal(d), torch.bfloat16)
        self.kw, self.kw64 = rounded(1 + 0.2 * rng.standard_normal(d), torch.bfloat16)
        self.lens = np.array([prompt - 13 * b for b in range(B)], np.int32)      # ragged prompts
        self.rows = {n: rounded(rng.standard_normal((B, n_rows, (H + 2 * Hkv) * d)), torch.bfloat16)[0]
                     for n, n_rows in [("prompt", prompt)] + [(k, bl) for k in range(steps)]}

    def split(self, rows):
        B, n, _ = rows.shape
        H, Hkv, d = self.H, self.Hkv, self.d
        q, k, v = rows.split([H * d, Hkv * d, Hkv * d], -1)
        return q.view(B, n, H, d).transpose(1, 2), k.view(B, n, Hkv, d).transpose(1, 2), v.view(B, n, Hkv, d).transpose(1, 2)

    def append(self, rows, starts, n_rows=None, lens=None):
        _, k, v = self.split(rows)
        dd.dd_paged_cache_append(self.Kc, self.Vc, k, v, self.table, starts, kv_lens=lens, n_rows=n_rows, k_scale=self.ks, v_scale=self.vs, k_weight=self.kw,
                                 inv_freq=self.f)

    def attend(self, rows, positions, lens, O=None):
        q, _, _ = self.split(rows)
        q, _ = dd.dd_qk_norm_rope(q, q_weight=self.qw, inv_freq=self.f, positions=positions)
        return q, dd.dd_paged_attention(q, self.Kc, self.Vc, self.table, lens, k_scale=self.ks, v_scale=self.vs, O=O)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_prompt_then_blocks(cache):
    s = Served(cache=cache)
    starts = s.lens.copy()
    s.append(s.rows["prompt"], ints(np.zeros(s.B)), n_rows=ints(s.lens))
    fresh = {b: [host(x)[b, :, :s.lens[b]] for x in s.split(s.rows["prompt"])[1:]] for b in range(s.B)}
    for k in range(2):
        for again in range(2):                               # a block is drafted twice: its rows replace those of the step before
            rows = s.rows[k] if again else s.rows[k].flip(1).contiguous()
            pos = starts[:, None] + np.arange(s.bl)[None]
            s.append(rows, ints(starts), lens=ints(starts + again * s.bl))
            q, O = s.attend(rows, ints(pos), ints(starts + s.bl))
            # the cache holds the rows to half a step of its type, and the attention is that of what it holds
            values = (lambda c: E4M3[codes_of(c)]) if cache == "fp8" else host
            want, A = paged.paged_attention(host(q), values(s.Kc), values(s.Vc), None if s.ks is None else host(s.ks), None if s.vs is None else host(s.vs),
                                            s.table.cpu().numpy(), starts + s.bl)
            assert (np.abs(host(O) - want) <= attention_tolerance(want, A)).all()
        for b in range(s.B):
            fresh[b] = [np.concatenate([a, host(x)[b]], 1) for a, x in zip(fresh[b], s.split(s.rows[k])[1:])]
        starts = starts + s.bl
    # end to end against attention on the rows themselves: e4m3 storage is off by 2^-4 of an element at most, bf16 by 2^-8
    half = 2.0 ** -4 if cache == "fp8" else 2.0 ** -8
    table = s.table.cpu().numpy()
    for b in range(s.B):
        n = int(starts[b])
        k = paged.norm_rope(fresh[b][0][None], s.kw64, 1e-6, s.freq, np.arange(n)[None], False)[0]
        for g in range(s.Hkv):
            for got, want, scale in ((s.Kc, k, s.ks), (s.Vc.transpose(2, 3), fresh[b][1], s.vs)):
                page = (E4M3[codes_of(got.contiguous())] if cache == "fp8" else host(got))[table[b], g]
                if scale is not None:
                    page = page * host(scale)[table[b], g][:, None, None]
                top = np.abs(want[g]).max()
                # (below 2^-6 of the scale steps are 2^-9 of it, and codes may have been rounded a second time in a larger scale; scale <= 2 top / 448)
                tol = 2 * half * np.abs(want[g]) + (2.0 ** -9 * 4 * top / 448 if cache == "fp8" else 0) + 2 * ROW_FAST * top
                assert (np.abs(page.reshape(-1, s.d)[:n] - want[g]) <= tol).all()


def test_verifier_takes_the_same_rows():
    # the dense path: queries and keys through dd_qk_norm_rope into dd_bidir_attention, against the paged path on the same rows
    import torch
    s = Served(B=2, cache="bf16", prompt=200, steps=0)
    q, k, v = s.split(s.rows["prompt"])
    Q, K = dd.dd_qk_norm_rope(q, k, q_weight=s.qw, k_weight=s.kw, inv_freq=s.f)
    dense = dd.dd_bidir_attention(Q, K, v.contiguous())
    s.append(s.rows["prompt"], ints([0, 0]))
    pos = np.broadcast_to(np.arange(200), (2, 200))
    q2, O = s.attend(s.rows["prompt"], ints(pos), ints([200, 200]))
    assert torch.equal(Q, q2)
    want, A = paged.paged_attention(host(q2), host(s.Kc), host(s.Vc), None, None, s.table.cpu().numpy(), [200, 200])
    assert (np.abs(host(O) - want) <= attention_tolerance(want, A)).all()
    assert (np.abs(host(dense) - want) <= attention_tolerance(want, A)).all()
    assert_rows(host(K), paged.norm_rope(host(k), s.kw64, 1e-6, s.freq, pos, False), 2.0 ** -8, ROW_FAST)


def test_graph_replays_match_eager_calls():
    import torch
    s = Served(B=2, prompt=700, bl=8, steps=1)
    s.append(s.rows["prompt"], ints([0, 0]), n_rows=ints(s.lens))
    starts, lens = ints(s.lens), ints(s.lens + s.bl)
    pos = starts[:, None] + torch.arange(s.bl, dtype=torch.int32, device="cuda")
    O = torch.zeros((s.B, s.H, s.bl, s.d), dtype=torch.bfloat16, device="cuda")
    rows = s.rows[0]

    def step():
        s.append(rows, starts)
        s.attend(rows, pos, lens, O=O)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (O, s.Kc, s.Vc, s.ks, s.vs)]
    graph = capture_step(step)
    for rep in range(4):
        O.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (O, s.Kc, s.Vc, s.ks, s.vs))), f"replay {rep}"
        step()
        torch.cuda.synchronize()
    # new rows and lengths in the same buffers: the graph goes by what they hold
    rows.copy_(rows.flip(1))
    starts -= 3
    lens -= 3
    pos -= 3
    kept = [t.clone() for t in (s.Kc, s.Vc, s.ks, s.vs)]
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (O, s.Kc, s.Vc, s.ks, s.vs)]
    for rep in range(3):
        for t, k in zip((s.Kc, s.Vc, s.ks, s.vs), kept):
            t.copy_(k)
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (O, s.Kc, s.Vc, s.ks, s.vs))), f"replay {rep} on other inputs"


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
def test_two_graphs_at_once(cache):
    # two captured steps whose attention is split, each with a scratch of its own, replayed on two streams between eager calls on a third
    import torch
    served = [Served(B=1, prompt=2300 + 700 * k, bl=3, steps=1, seed=k, cache=cache) for k in range(2)]
    graphs, want = [], []
    for s in served:
        s.append(s.rows["prompt"], ints([0]))
        s.args, s.O = (ints(s.lens), ints(s.lens + 3), ints(s.lens[:, None] + np.arange(3))), torch.zeros((1, s.H, 3, s.d), dtype=torch.bfloat16, device="cuda")
        assert dd.dd_paged_attention_workspace_bytes(3, 1, s.H, s.Hkv, s.d, 64, s.table.shape[1], dd.FP8_E4M3 if cache == "fp8" else dd.BF16) > 0

        def step(s=s, O=s.O):
            s.append(s.rows[0], s.args[0])
            s.attend(s.rows[0], s.args[2], s.args[1], O=O)

        step()
        torch.cuda.synchronize()
        want.append(s.O.clone())
        graphs.append(capture_step(step))
    streams = [torch.cuda.Stream() for _ in graphs]
    for rep in range(5):
        for s in served:
            s.O.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        q = dd.dd_qk_norm_rope(served[0].split(served[0].rows[0])[0], q_weight=served[0].qw, inv_freq=served[0].f, positions=served[0].args[2])[0]
        eager = dd.dd_paged_attention(q, served[1].Kc, served[1].Vc, served[1].table, ints([1999]), k_scale=served[1].ks, v_scale=served[1].vs)
        torch.cuda.synchronize()
        assert all(torch.equal(s.O, w) for s, w in zip(served, want)), f"replay {rep}"
        again = dd.dd_paged_attention(q, served[1].Kc, served[1].Vc, served[1].table, ints([1999]), k_scale=served[1].ks, v_scale=served[1].vs)
        assert torch.equal(eager, again)


def test_streams_side_by_side():
    import torch
    batches = [Served(B=1, prompt=900, bl=4, steps=1, seed=k) for k in range(3)]
    want = []
    for s in batches:
        s.append(s.rows["prompt"], ints([0]))
        s.args = ints(s.lens), ints(s.lens + 4), ints(s.lens[:, None] + np.arange(4))
        s.append(s.rows[0], s.args[0])
        want.append(s.attend(s.rows[0], s.args[2], s.args[1])[1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    got = [[] for _ in batches]
    for _ in range(5):
        for s, stream, to in zip(batches, streams, got):
            with torch.cuda.stream(stream):
                s.append(s.rows[0], s.args[0])
                to.append(s.attend(s.rows[0], s.args[2], s.args[1])[1])
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for w, os in zip(want, got) for o in os)


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("n,P,lens", [(1, 64, [700, 3]), (33, 16, [50, 81]), (70, 128, [130, 1])])
def test_nothing_else_is_written(cache, n, P, lens):
    import torch
    g = Guarded()
    B, H, Hkv, d = 2, 4, 2, 128
    per = -(-max(lens) // P) + -(-n // P) + 1
    pages = B * per
    t = torch.uint8 if cache == "fp8" else torch.bfloat16
    Kc, Vc = g.empty((pages, Hkv, P, d), t), g.empty((pages, Hkv, d, P), t)
    Kc.zero_(), Vc.zero_()
    ks, vs = (g.empty((pages, Hkv), torch.float32).fill_(1), g.empty((pages, Hkv), torch.float32).fill_(1)) if cache == "fp8" else (None, None)
    x = torch.randn((B, n, (H + 2 * Hkv) * d), device="cuda").bfloat16()
    q, k, v = (y.view(B, n, -1, d).transpose(1, 2) for y in x.split([H * d, Hkv * d, Hkv * d], -1))
    Qo, Ko, O = g.empty((B, H, n, d), torch.bfloat16), g.empty((B, Hkv, n, d), torch.bfloat16), g.empty((B, H, n, d), torch.bfloat16)
    table = ints(np.arange(pages).reshape(B, per)[:, ::-1])
    starts = ints(lens)
    f = dev((10000.0 ** (-np.arange(32) / 32)).astype(np.float32))
    kept = table.clone(), starts.clone(), x.clone()
    dd.dd_qk_norm_rope(q, k, inv_freq=f, Qo=Qo, Ko=Ko)
    dd.dd_paged_cache_append(Kc, Vc, k, v, table, starts, k_scale=ks, v_scale=vs, inv_freq=f)
    need = dd.dd_paged_attention_workspace_bytes(n, B, H, Hkv, d, P, per, dd.FP8_E4M3 if cache == "fp8" else dd.BF16)
    with dd.fixed_workspace(guarded_workspace(g, need)):
        dd.dd_paged_attention(Qo, Kc, Vc, table, starts + n, k_scale=ks, v_scale=vs, O=O)
    g.check(f"{cache} n {n} P {P}")
    assert all(torch.equal(a, b) for a, b in zip(kept, (table, starts, x)))
    # of the cache, the rows' slots alone (zeros elsewhere, which any scale leaves as they are)
    held = torch.zeros((pages, P), dtype=torch.bool, device="cuda")
    for b in range(B):
        p = torch.arange(lens[b], lens[b] + n, device="cuda")
        held[table[b].long()[p // P], p % P] = True
    assert not Kc.masked_fill(held[:, None, :, None], 0).any() and not Vc.masked_fill(held[:, None, None, :], 0).any()
    assert bool(Kc[held.nonzero()[0, 0]].any()) and O.isfinite().all()
