"""The calls of a batch that shares prompts and drafts ahead, together as a serving loop makes them: pages for the drafted rows, rows into the
pages, attention over prompt and own positions, the drafts against the verifier, pages of what was turned down back to the pool."""
import numpy as np
import pytest

import paper_2604_05250_amd as dd
from oracle import draft, paged
from paper_2604_05250_amd.step import capture_step
from _paged import E4M3, attention_tolerance, codes_of, dev, host, ints, rounded
from test_gpu_verify_draft import NEAR

pytestmark = pytest.mark.gpu


class Loop:
    """Prompts of several groups of sequences, and what the sequences hold for themselves, on one pool of pages."""

    def __init__(self, groups=(3, 2), prompts=(150, 90), H=8, Hkv=2, d=128, P=16, n=6, room=80, V=512, cache="fp8", seed=0):
        import torch
        rng = np.random.default_rng(seed)
        self.groups, self.prompts, self.H, self.Hkv, self.d, self.P, self.n, self.V = groups, prompts, H, Hkv, d, P, n, V
        self.B, self.G = sum(groups), len(groups)
        pages = sum(-(-x // P) for x in prompts) + self.B * -(-room // P)
        t = torch.uint8 if cache == "fp8" else torch.bfloat16
        self.Kc, self.Vc = torch.zeros((pages, Hkv, P, d), dtype=t, device="cuda"), torch.zeros((pages, Hkv, d, P), dtype=t, device="cuda")
        self.ks = self.vs = None
        if cache == "fp8":
            self.ks, self.vs = torch.ones((pages, Hkv), device="cuda"), torch.ones((pages, Hkv), device="cuda")
        self.pool, self.free = ints(rng.permutation(pages)), ints([pages])
        self.prefix_table = ints(np.full((self.G, -(-max(prompts) // P)), -1))
        self.table = ints(np.full((self.B, -(-room // P)), -1))
        self.starts = ints(np.concatenate([[0], np.cumsum(groups)]))
        self.f = dev((10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32))
        self.offset = ints(np.repeat(prompts, groups))       # a sequence's positions begin behind its prompt
        # the prompts: places, then rows, keys turned by position
        self.prefix_lens, positions, _ = dd.dd_paged_resize(self.prefix_table, self.pool, self.free, ints(np.zeros(self.G)), ints(prompts), P, n=max(prompts))
        rows = rounded(rng.standard_normal((self.G, max(prompts), 2 * Hkv * d)), torch.bfloat16)[0]
        k, v = (x.view(self.G, -1, Hkv, d).transpose(1, 2) for x in rows.split(Hkv * d, -1))
        dd.dd_paged_cache_append(self.Kc, self.Vc, k, v, self.prefix_table, ints(np.zeros(self.G)), n_rows=self.prefix_lens, k_scale=self.ks, v_scale=self.vs, inv_freq=self.f)
        self.lens = ints(np.zeros(self.B))
        self.O = torch.zeros((self.B, H, n, d), dtype=torch.bfloat16, device="cuda")
        self.out = (torch.zeros((self.B, n + 1), dtype=torch.int32, device="cuda"), torch.zeros(self.B, dtype=torch.int32, device="cuda"),
                    torch.zeros((self.B, n), device="cuda"))
        self.grown, self.positions = torch.zeros_like(self.lens), torch.zeros((self.B, n), dtype=torch.int32, device="cuda")
        self.slots = torch.zeros_like(self.positions)
        self.wanted = torch.zeros_like(self.lens)
        self.feed(rng)

    def feed(self, rng):
        """what a model would bring: rows of a projection, drafts, logits, random numbers"""
        import torch
        B, n, V = self.B, self.n, self.V
        rows = rounded(rng.standard_normal((B, n, (self.H + 2 * self.Hkv) * self.d)), torch.bfloat16)[0]
        d = 3 * rng.standard_normal((B, n + 1, V))
        lv, ld = rounded(d + rng.standard_normal(d.shape), torch.bfloat16)[0], rounded(d[:, :n], torch.bfloat16)[0]
        p = host(ld)
        x = np.array([[rng.choice(V, p=draft.probabilities(p[b, i], 1.0)) for i in range(n)] for b in range(B)])
        new = rows, lv, ld, ints(x), dev(rng.random((B, n + 1)).astype(np.float32))
        if not hasattr(self, "fed"):
            self.fed = new
        else:
            for a, b in zip(self.fed, new):
                a.copy_(b)

    def step(self):
        import torch
        rows, lv, ld, tokens, u = self.fed
        H, Hkv, d, n = self.H, self.Hkv, self.d, self.n
        q, k, v = (x.view(self.B, n, -1, d).transpose(1, 2) for x in rows.split([H * d, Hkv * d, Hkv * d], -1))
        torch.add(self.lens, n, out=self.wanted)
        dd.dd_paged_resize(self.table, self.pool, self.free, self.lens, self.wanted, self.P, n, out_lens=self.grown, positions=self.positions, slots=self.slots)
        self.q, self.k = dd.dd_qk_norm_rope(q, k, inv_freq=self.f, positions=self.positions + self.offset[:, None])
        dd.dd_paged_cache_append(self.Kc, self.Vc, self.k, v, self.table, self.lens, n_rows=self.grown - self.lens, k_scale=self.ks, v_scale=self.vs)
        dd.dd_paged_attention_shared(self.q, self.Kc, self.Vc, self.prefix_table, self.prefix_lens, self.starts, self.table, self.grown, k_scale=self.ks, v_scale=self.vs, O=self.O)
        dd.dd_verify_draft(lv, ld, tokens, u, n_draft=self.grown - self.lens, out_tokens=self.out[0], out_accepted=self.out[1], out_chances=self.out[2])
        torch.add(self.lens, self.out[1], out=self.wanted)   # the rows of drafts that stand stay
        dd.dd_paged_resize(self.table, self.pool, self.free, self.grown, self.wanted, self.P, out_lens=self.lens)

    def state(self):
        return [t for t in (self.Kc, self.Vc, self.ks, self.vs, self.pool, self.free, self.table, self.lens, self.O, *self.out, self.slots) if t is not None]


@pytest.mark.parametrize("cache", ["fp8", "bf16"])
@pytest.mark.parametrize("room", [80, 24])
def test_steps_of_a_loop(cache, room):
    # (room 24: sequences run out of pages, and stay as they are for want of them)
    loop, rng = Loop(cache=cache, room=room), np.random.default_rng(9)
    refused = 0
    for _ in range(7):
        before = loop.lens.cpu().numpy()
        loop.step()
        grown, lens, free = loop.grown.cpu().numpy(), loop.lens.cpu().numpy(), int(loop.free)
        refused += int((grown == before).sum())
        # every page is in one place: a prompt's, a sequence's or the pool's
        held = [x for t in (loop.prefix_table, loop.table) for x in t.flatten().tolist() if x >= 0] + loop.pool.tolist()[:free]
        assert sorted(held) == list(range(len(loop.Kc)))
        # the drafts, by the oracle
        want = draft.verify_draft(host(loop.fed[1]), host(loop.fed[2]), loop.fed[3].cpu().numpy(), host(loop.fed[4]), n_draft=grown - before)
        sure = want[3] > NEAR
        assert sure.any() and np.array_equal(loop.out[0].cpu().numpy()[sure], want[0][sure]) and np.array_equal(lens, before + loop.out[1].cpu().numpy())
        # the attention, on what the cache holds; tables as they were before pages went back: from the slots
        table = loop.table.cpu().numpy().copy()
        for b in range(loop.B):
            for p, s in zip(loop.positions[b].tolist(), loop.slots[b].tolist()):
                assert (s >= 0) == (p < grown[b])
                if s >= 0:
                    table[b, p // loop.P] = s // loop.P
                    assert s % loop.P == p % loop.P
        values = (lambda c: E4M3[codes_of(c)]) if cache == "fp8" else host
        O, A = paged.paged_attention_shared(host(loop.q), values(loop.Kc), values(loop.Vc), None if loop.ks is None else host(loop.ks), None if loop.vs is None else host(loop.vs),
                                            loop.prefix_table.cpu().numpy(), loop.prefix_lens.tolist(), loop.starts.tolist(), table, grown)
        assert (np.abs(host(loop.O) - O) <= attention_tolerance(O, A)).all()
        if cache == "bf16":                                  # a row is where its slot says
            for b in range(loop.B):
                for r, s in enumerate(loop.slots[b].tolist()):
                    if s >= 0:
                        assert np.array_equal(host(loop.Kc)[s // loop.P, :, s % loop.P], host(loop.k)[b, :, r])
        loop.feed(rng)
    assert (refused > 0) == (room == 24)


def test_steps_as_a_graph():
    import torch
    loop, rng = Loop(seed=4), np.random.default_rng(5)
    kept = [t.clone() for t in loop.state()]
    graph = capture_step(loop.step)
    for t, k in zip(loop.state(), kept):
        t.copy_(k)
    for rep in range(5):
        loop.feed(rng)
        before = [t.clone() for t in loop.state()]
        loop.step()
        torch.cuda.synchronize()
        want = [t.clone() for t in loop.state()]
        for t, k in zip(loop.state(), before):
            t.copy_(k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, loop.state())), f"replay {rep}"
