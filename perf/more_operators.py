"""The operators of a batch that shares prompts and drafts ahead, on the sizes that their callers use.

A case is one of three kinds:
  tables  dd_paged_resize: pages, positions and slots of sequences that grow, shrink and end
  shared  dd_paged_attention_shared: attention of a batch whose sequences share long prefixes, over pages of bf16 or e4m3
  verify  dd_verify_draft: drafted tokens against the verifier's probabilities, with given random numbers
With `own` false, run() computes them in plain torch operations; with `own` true, it calls this package.
"""
import math

import torch

own = False

E4M3_MAX = 448.0


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one token of each sequence of a serving batch taken back, one more drafted: nothing but latency
        _tables("tables_token_b16", B=16, n=1, N=2048, page=64, kind_of="grow"),
        # an odd batch in mid-flight: some grow by up to a block, some give drafted rows back, some end, some are admitted
        _tables("tables_mixed_b57", B=57, n=64, N=1237, page=16, kind_of="mixed"),
        # a large batch ends, and as many prompts are admitted at once
        _tables("tables_prompts_b64_n2048", B=64, n=2048, N=2048, page=16, kind_of="admit"),
        # few answers to a short prompt, one token each: latency
        _shared("shared_fp8_token_b4_p1024", groups=[4], H=32, Hkv=8, n=1, prefix=1024, N=64, d=128, page=64, cache="fp8"),
        # a serving batch under one long prompt
        _shared("shared_fp8_token_b16_p4096", groups=[16], H=32, Hkv=8, n=1, prefix=4096, N=512, d=128, page=64, cache="fp8"),
        # three prompts of odd length and as many odd groups, small heads, bf16 pages of 16
        _shared("shared_bf16_token_b21_p1237", groups=[7, 12, 2], H=28, Hkv=4, n=1, prefix=1237, N=200, d=64, page=16, cache="bf16"),
        # many answers to a document
        _shared("shared_fp8_token_b64_p32768", groups=[64], H=32, Hkv=8, n=1, prefix=32768, N=256, d=128, page=64, cache="fp8"),
        # the drafter's blocks of a batch with one prompt: compute bound
        _shared("shared_fp8_block_b16_p2048", groups=[16], H=32, Hkv=8, n=64, prefix=2048, N=256, d=128, page=64, cache="fp8"),
        # the checkable size: fp32 logits, an odd batch, drafts of different lengths, some sequences at temperature 0
        _verify("verify_f32_b5_k5", B=5, n=5, V=1024, dtype="f32", ragged=True, temperature="mixed"),
        # one sequence, four drafted tokens: latency
        _verify("verify_bf16_b1_k4", B=1, n=4, V=126464, dtype="bf16"),
        # a drafter that proposes without probabilities
        _verify("verify_bf16_b32_k4_sure", B=32, n=4, V=152064, dtype="bf16", drafter=False, temperature="warm"),
        # a serving batch that drafts eight ahead: the largest stream of bytes
        _verify("verify_bf16_b64_k8", B=64, n=8, V=126464, dtype="bf16"),
    ]


def draw(rng):
    kind = rng.choice(["tables", "shared", "shared", "verify", "verify"])
    if kind == "tables":
        page, B = rng.choice([16, 32, 64, 128]), _log_int(rng, 1, 256)
        N = _log_int(rng, page, 4096)
        n = min(N, _log_int(rng, 1, 2048))
        while B * n > 64 * 2048:
            n = max(1, n // 2)
        return _tables(None, B=B, n=n, N=N, page=page, kind_of=rng.choice(["grow", "mixed", "admit", "mixed"]), scarce=rng.random() < 0.3)
    if kind == "shared":
        d = 64 if rng.random() < 0.25 else 128
        H, Hkv = rng.choice([(4, 2), (28, 4), (32, 32)] if d == 64 else [(32, 32), (32, 8), (28, 4), (16, 2)])
        groups = [_log_int(rng, 1, 48) for _ in range(rng.choice([1, 1, 1, 2, 3, 5]))]
        n = rng.choice([1, 1, 1, 2, 8, 16, 32, 64])
        prefix, N = _log_int(rng, 16, 32768), _log_int(rng, 1, 1024)
        while sum(groups) > 64:
            groups = [max(1, m // 2) for m in groups]
        while sum(groups) * H * n * (prefix + N) * d > 64 * 32 * 32768 * 128:
            prefix, N = max(16, prefix // 2), max(1, N // 2)
        while len(groups) * Hkv * prefix * d > 8 * 32768 * 128:                # no more bytes of prefixes than the largest listed call has
            prefix = prefix // 2
        return _shared(None, groups=groups, H=H, Hkv=Hkv, n=n, prefix=prefix, N=N, d=d, page=rng.choice([16, 32, 64, 64, 128]),
                       cache=rng.choice(["fp8", "fp8", "bf16"]), bare=rng.random() < 0.25)
    B, n, dtype = _log_int(rng, 1, 64), rng.randint(1, 8), rng.choice(["bf16", "bf16", "f32"])
    V = 8 * _log_int(rng, 128, 19008)
    while B * (2 * n + 1) * V * (2 if dtype == "bf16" else 4) > 64 * 17 * 126464 * 2:
        B = max(1, B // 2)
    return _verify(None, B=B, n=n, V=V, dtype=dtype, ragged=rng.random() < 0.5, drafter=rng.random() < 0.75, bonus=rng.random() < 0.8,
                   temperature=rng.choice(["one", "warm", "mixed"]))


def _tables(name, B, n, N, page, kind_of, scarce=False):
    return _named(name, dict(kind="tables", B=B, n=n, N=N, page=page, kind_of=kind_of, scarce=scarce))


def _shared(name, groups, H, Hkv, n, prefix, N, d, page, cache, bare=False):
    """bare: some sequences have nothing of their own yet, and the last of several groups has no prefix."""
    return _named(name, dict(kind="shared", groups=",".join(map(str, groups)), B=sum(groups), H=H, Hkv=Hkv, n=n, prefix=prefix, N=N, d=d, page=page, cache=cache,
                             bare=bare))


def _verify(name, B, n, V, dtype, ragged=False, drafter=True, bonus=True, temperature="one"):
    return _named(name, dict(kind="verify", B=B, n=n, V=V, dtype=dtype, ragged=ragged, drafter=drafter, bonus=bonus, temperature=temperature))


def _named(name, case):
    return case if name is None else dict(case, name=name)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _groups(case):
    """How many sequences each prefix has."""
    return [int(m) for m in case["groups"].split(",")]


def _own_lengths(case):
    """The positions that each sequence of a shared case holds for itself: ragged, N at most."""
    N = case["N"]
    return [0 if case["bare"] and b % 3 == 2 else max(1, N - (b * 41) % (N // 2 + 1)) for b in range(case["B"])]


def _prefix_lengths(case):
    """The prefixes' lengths: the first is the longest."""
    p, G = case["prefix"], len(_groups(case))
    return [0 if case["bare"] and g > 0 and g == G - 1 else p - (g * 211) % (p // 2 + 1) for g in range(G)]


def _drafted(case):
    n = case["n"]
    return [n - (b * 5) % (n + 1) if case["ragged"] else n for b in range(case["B"])]


def _steps(case):
    """[(length at first, length in between)] of every sequence of a tables case."""
    n, N, out = case["n"], case["N"], []
    for b in range(case["B"]):
        full = max(n, N - (b * 97) % (N // 4 + 1))
        rows, turn = 1 + (b * 13) % n, b % 7
        if case["kind_of"] == "admit":
            out.append((min(full, n), 0))
        elif case["kind_of"] == "grow":
            out.append((full, full - n))
        elif turn == 1:
            out.append((full, full - rows))
        elif turn == 4:
            out.append((full, 0))
        elif turn == 6:
            out.append((0, rows))
        else:
            out.append((full - n, full - n + rows))
    return out


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"tables": _prepare_tables, "shared": _prepare_shared, "verify": _prepare_verify}[case["kind"]](case, g)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_tables(case, g):
    page, steps = case["page"], _steps(case)
    width = -(-case["N"] // page) + 1
    held = [-(-a // page) for a, _ in steps]
    wanted = sum(max(0, -(-w // page) - h) for h, (_, w) in zip(held, steps))
    back = sum(max(0, h - -(-w // page)) for h, (_, w) in zip(held, steps))
    free = max(0, wanted - back) // 2 if case["scarce"] else wanted + 5   # a pool that does not serve everyone, or one that does
    pages = sum(held) + free
    order = torch.randperm(max(1, pages), generator=g, device="cuda").to(torch.int32)
    table = torch.full((case["B"], width), -1, dtype=torch.int32, device="cuda")
    rows = torch.arange(width, device="cuda")
    first = torch.tensor([sum(held[:b]) for b in range(case["B"])], device="cuda").unsqueeze(1)
    mine = rows < torch.tensor(held, device="cuda").unsqueeze(1)
    table[mine] = order[(first + rows)[mine]]
    stack = torch.full((max(1, pages),), -1, dtype=torch.int32, device="cuda")
    stack[:free] = order[sum(held):sum(held) + free]
    return {"case": dict(case), "table": table, "free_pages": stack, "num_free": _ints([free]),
            "lens": _ints([a for a, _ in steps]), "between": _ints([w for _, w in steps])}


def _prepare_shared(case, g):
    B, H, Hkv, n, d, page = (case[k] for k in ("B", "H", "Hkv", "n", "d", "page"))
    G = len(_groups(case))
    shared, per = -(-case["prefix"] // page), -(-case["N"] // page)
    pages = G * shared + B * per + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    st = {"case": dict(case), "prefix_table": order[:G * shared].view(G, shared), "block_table": order[G * shared:G * shared + B * per].view(B, per),
          "prefix_lens": _ints(_prefix_lengths(case)), "kv_lens": _ints(_own_lengths(case)),
          "group_starts": _ints([sum(_groups(case)[:i]) for i in range(G + 1)])}
    kshape, vshape = (pages, Hkv, page, d), (pages, Hkv, d, page)
    if case["cache"] == "fp8":
        st["Kc"] = (70 * _normal(g, *kshape)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        st["Vc"] = (70 * _normal(g, *vshape)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        st["k_scale"] = torch.exp2(torch.randint(-7, -5, (pages, Hkv), generator=g, device="cuda").float())
        st["v_scale"] = torch.exp2(torch.randint(-7, -5, (pages, Hkv), generator=g, device="cuda").float())
    else:
        st["Kc"], st["Vc"] = _normal(g, *kshape).bfloat16(), _normal(g, *vshape).bfloat16()
        st["k_scale"] = st["v_scale"] = None
    st["Q"] = (1.5 * _normal(g, B, H, n, d)).bfloat16()
    st["O"] = torch.empty_like(st["Q"])
    return st


def _prepare_verify(case, g):
    B, n, V = case["B"], case["n"], case["V"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    rows = n + (1 if case["bonus"] else 0)
    drafter = 3.0 * _normal(g, B, rows, V)                                # as the drafter's logits are in the benchmark's configurations
    st = {"case": dict(case), "logits_v": (drafter + _normal(g, B, rows, V)).to(dt)}
    if case["temperature"] == "one":
        st["temperature"] = None
        t = torch.ones(B, device="cuda")
    else:
        t = 0.5 + torch.rand(B, generator=g, device="cuda")
        if case["temperature"] == "mixed":
            t[1::3] = 0.0
        st["temperature"] = t
    logits_d = drafter[:, :n].to(dt)
    noise = -torch.log(-torch.log(torch.rand((B, n, V), generator=g, device="cuda").clamp(1e-30, 1 - 2.0 ** -24)))
    drawn = (logits_d.float() + t.view(B, 1, 1) * noise).argmax(-1)       # a draw from the drafter's distribution at that temperature
    st["tokens"] = drawn.to(torch.int32)
    st["logits_d"] = logits_d.contiguous() if case["drafter"] else None
    st["uniforms"] = torch.rand((B, n + 1), generator=g, device="cuda")
    st["n_draft"] = _ints(_drafted(case)) if case["ragged"] else None
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if own:
        return {"tables": _own_tables, "shared": _own_shared, "verify": _own_verify}[case["kind"]](st, case)
    return {"tables": _plain_tables, "shared": _plain_shared, "verify": _plain_verify}[case["kind"]](st, case)


def _own_tables(st, case):
    """Away from the lengths and back to them, with the places of the rows that come: a table that a call gets wrong does not come back."""
    import paper_2604_05250_amd as dd
    between, _, _ = dd.dd_paged_resize(st["table"], st["free_pages"], st["num_free"], st["lens"], st["between"], case["page"])
    lens, positions, slots = dd.dd_paged_resize(st["table"], st["free_pages"], st["num_free"], between, st["lens"], case["page"], case["n"])
    return _tables_out(st, between, lens, positions, slots)


def _own_shared(st, case):
    import paper_2604_05250_amd as dd
    return {"O": dd.dd_paged_attention_shared(st["Q"], st["Kc"], st["Vc"], st["prefix_table"], st["prefix_lens"], st["group_starts"], st["block_table"],
                                              st["kv_lens"], k_scale=st["k_scale"], v_scale=st["v_scale"], O=st["O"])}


def _own_verify(st, case):
    import paper_2604_05250_amd as dd
    tokens, accepted, chances = dd.dd_verify_draft(st["logits_v"], st["logits_d"], st["tokens"], st["uniforms"], temperature=st["temperature"],
                                                   n_draft=st["n_draft"])
    return {"tokens": tokens, "accepted": accepted, "chances": chances}


def _tables_out(st, between, lens, positions, slots):
    return {"table": st["table"], "free_pages": st["free_pages"], "num_free": st["num_free"], "between": between, "lens": lens, "positions": positions,
            "slots": slots}


# ---------------------------------------------------------------- the plain forms
def _plain_tables(st, case):
    between, _, _ = _resize(st, st["lens"], st["between"], case["page"], 0)
    lens, positions, slots = _resize(st, between, st["lens"], case["page"], case["n"])
    return _tables_out(st, between, lens, positions, slots)


def _resize(st, lens, new_lens, page, n):
    table, stack, count = st["table"], st["free_pages"], st["num_free"]
    B, width = table.shape
    lens, want = lens.long(), new_lens.long()
    have, need = (lens + page - 1) // page, (want + page - 1) // page
    fits = need <= width
    back = (have - need).clamp(min=0)
    take = torch.where(fits, (need - have).clamp(min=0), 0)
    pushed = back.cumsum(0)
    top = count.long() + pushed[-1]                                       # what is free once the pages that come back are there
    end = take.cumsum(0)
    granted = fits & ((take == 0) | (end <= top))
    column = torch.arange(width, device=table.device)
    # pages that come back: the first sequence's first one ends up on top
    gone = (column >= need.unsqueeze(1)) & (column < have.unsqueeze(1))
    rank = (pushed - back).unsqueeze(1) + column - need.unsqueeze(1)
    more = torch.cat([stack, stack[:1]])                                  # one entry behind the end for what goes nowhere
    more.scatter_(0, torch.where(gone, top - 1 - rank, len(stack)).flatten(), table.flatten())
    stack.copy_(more[:-1])
    table.masked_fill_(gone, -1)
    # pages that are taken: the first sequence's first one from the top
    new = (column >= have.unsqueeze(1)) & (column < need.unsqueeze(1)) & granted.unsqueeze(1)
    rank = (end - take).unsqueeze(1) + column - have.unsqueeze(1)
    table.copy_(torch.where(new, stack[torch.where(new, top - 1 - rank, 0)], table))
    count.copy_(top - torch.where(granted, take, 0).sum())
    out = torch.where(granted, want, lens)
    positions = lens.unsqueeze(1) + torch.arange(n, device=table.device)
    at = table.long().gather(1, (positions // page).clamp(max=width - 1))
    slots = torch.where(positions < out.unsqueeze(1), at * page + positions % page, -1)
    return out.int(), positions.int(), slots.int()


def _held(cache, scale, ids):
    """The values of pages, [..., Hkv, page, d] or [..., Hkv, d, page]."""
    if scale is None:
        return cache[ids].float()
    return cache.view(torch.uint8)[ids].view(cache.dtype).float() * scale[ids][..., None, None]


def _plain_shared(st, case):
    """The prefix's scores of a group at once, the own ones per sequence, one softmax over both."""
    B, H, Hkv, n, d = (case[k] for k in ("B", "H", "Hkv", "n", "d"))
    R, scale = H // Hkv * n, 1.0 / math.sqrt(d)
    Q = st["Q"].float().view(B, Hkv, R, d)
    ids = st["block_table"].long()
    K = _held(st["Kc"], st["k_scale"], ids).permute(0, 2, 4, 1, 3).reshape(B * Hkv, d, -1)
    V = _held(st["Vc"], st["v_scale"], ids).permute(0, 2, 1, 4, 3).reshape(B * Hkv, -1, d)
    S = torch.bmm(Q.view(B * Hkv, R, d), K) * scale
    hidden = (torch.arange(S.shape[-1], device="cuda") >= st["kv_lens"].unsqueeze(1)).repeat_interleave(Hkv, 0).unsqueeze(1)
    S = S.masked_fill(hidden, -math.inf)
    m = S.amax(-1).view(B, Hkv, R)
    starts, heads = 0, []
    for g, count in enumerate(_groups(case)):
        ids = st["prefix_table"][g].long()
        Kp = _held(st["Kc"], st["k_scale"], ids).permute(1, 3, 0, 2).reshape(Hkv, d, -1)
        Vp = _held(st["Vc"], st["v_scale"], ids).permute(1, 0, 3, 2).reshape(Hkv, -1, d)
        q = Q[starts:starts + count].transpose(0, 1).reshape(Hkv, count * R, d)
        s = torch.bmm(q, Kp) * scale
        s = s.masked_fill(torch.arange(s.shape[-1], device="cuda") >= st["prefix_lens"][g], -math.inf)
        heads.append((s, Vp, starts, count))
        starts += count
    O = torch.empty((B, Hkv, R, d), device="cuda")
    own_v = V.view(B, Hkv, -1, d)
    S = S.view(B, Hkv, R, -1)
    for s, Vp, first, count in heads:
        s_top = s.amax(-1).view(Hkv, count, R).transpose(0, 1)
        top = torch.maximum(m[first:first + count], s_top)
        top = torch.where(torch.isinf(top), 0.0, top)                     # a row without any key
        w = torch.exp(s - top.transpose(0, 1).reshape(Hkv, count * R, 1))
        v = torch.exp(S[first:first + count] - top.unsqueeze(-1))
        total = w.sum(-1).view(Hkv, count, R).transpose(0, 1) + v.sum(-1)
        x = torch.bmm(w, Vp).view(Hkv, count, R, d).transpose(0, 1)
        y = torch.bmm(v.reshape(count * Hkv, R, -1), own_v[first:first + count].reshape(count * Hkv, -1, d)).view(count, Hkv, R, d)
        O[first:first + count] = (x + y) / torch.where(total == 0, 1.0, total).unsqueeze(-1)
    return {"O": O.view(B, H, n, d).to(st["Q"].dtype)}


def _plain_verify(st, case):
    """In 64 bits: decisions stand next to borders."""
    B, n, V = case["B"], case["n"], case["V"]
    t = st["temperature"]
    t = torch.ones(B, dtype=torch.float64, device="cuda") if t is None else t.double()
    count = torch.full((B,), n, device="cuda") if st["n_draft"] is None else st["n_draft"].long()
    p = _softmax(st["logits_v"], t)
    x = st["tokens"].long().unsqueeze(-1)
    at_p = p[:, :n].gather(2, x).squeeze(-1)
    q = _softmax(st["logits_d"], t) if st["logits_d"] is not None else None
    at_q = torch.ones_like(at_p) if q is None else q.gather(2, x).squeeze(-1)
    chance = torch.where(at_q > at_p, at_p / torch.where(at_q > at_p, at_q, 1.0), (at_p > 0).double())
    u = st["uniforms"].double()
    row = torch.arange(n, device="cuda")
    refused = ~(u[:, :n] * at_q < at_p) & (row < count.unsqueeze(1))
    accepted = torch.minimum(torch.where(refused, row, n).amin(-1), count)
    which = torch.arange(B, device="cuda")
    r = p[which, accepted.clamp(max=p.shape[1] - 1)]
    turned = accepted < count                                             # a draft was turned down: from what p has more than q
    again = accepted.clamp(max=n - 1)
    minus = q[which, again] if q is not None else torch.zeros_like(r).scatter_(1, x[which, again], math.inf)
    left = (r - minus).clamp(min=0)
    r = torch.where((turned & (left.sum(-1) > 0)).unsqueeze(1), left, r)
    c = r.cumsum(-1)
    token = (c <= u[:, n:] * c[:, -1:]).sum(-1).clamp(max=V - 1)
    if not case["bonus"]:
        token = torch.where(turned, token, -1)
    out = torch.full((B, n + 1), -1, dtype=torch.long, device="cuda")
    out[:, :n] = torch.where(row < accepted.unsqueeze(1), st["tokens"].long(), -1)
    out.scatter_(1, accepted.unsqueeze(1), token.unsqueeze(1))
    chance = torch.where(row < count.unsqueeze(1), chance, 0.0)
    return {"tokens": out.int(), "accepted": accepted.int(), "chances": chance.float()}


def _softmax(logits, t):
    """Probabilities at each sequence's temperature; at 0 all of it on the first of the largest."""
    x = logits.double()
    top = x.amax(-1, keepdim=True)
    cold = (t == 0).view(-1, 1, 1)
    e = torch.exp((x - top) / torch.where(cold, 1.0, t.view(-1, 1, 1)))
    e = e / e.sum(-1, keepdim=True)
    column = torch.arange(x.shape[-1], device=x.device)
    first = torch.where(x == top, column, x.shape[-1]).amin(-1, keepdim=True)
    return torch.where(cold, (column == first).double(), e)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["kind"] == "tables":
        page, steps, n = case["page"], _steps(case), case["n"]
        moved = sum(abs(-(-a // page) - -(-w // page)) for a, w in steps)
        # away and back: lengths in and out, each page's entry in the table and in the stack read or written; positions and slots of the rows
        return {"bytes": 4 * (2 * 3 * case["B"] + 2 * 2 * moved + 2 * case["B"] * n), "flops": 0}
    if case["kind"] == "shared":
        B, H, Hkv, n, d, page = (case[k] for k in ("B", "H", "Hkv", "n", "d", "page"))
        el, scales = (1, 8 * Hkv) if case["cache"] == "fp8" else (2, 0)
        prefixes, owns = _prefix_lengths(case), _own_lengths(case)
        keys = sum(prefixes) + sum(owns)
        pages = sum(-(-t // page) for t in prefixes + owns)
        seen = sum(p * m for p, m in zip(prefixes, _groups(case))) + sum(owns)
        return {"bytes": 2 * 2 * B * H * n * d + 2 * keys * Hkv * d * el + pages * (scales + 4), "flops": 4 * H * n * d * seen}
    el = 2 if case["dtype"] == "bf16" else 4
    rows = sum(_drafted(case))
    logits = ((2 if case["drafter"] else 1) * rows + (case["B"] if case["bonus"] else 0)) * case["V"]
    return {"bytes": logits * el + 4 * case["B"] * (4 * case["n"] + 4), "flops": 3 * logits}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"tables": _exact_tables, "shared": _exact_shared, "verify": _exact_verify}[case["kind"]](st, case)


def _exact_tables(st, case):
    """Lists and loops: sequences one after the other."""
    page, width = case["page"], st["table"].shape[1]
    held = [[int(x) for x in row if x >= 0] for row in st["table"].tolist()]
    stack = st["free_pages"].tolist()
    free = stack[:int(st["num_free"])]

    def resize(lens, wanted, n):
        back, out, positions, slots = [], [], [], []
        for pages, w in zip(held, wanted):
            keep = -(-w // page)
            if keep < len(pages):
                back += pages[keep:]
                del pages[keep:]
        free.extend(reversed(back))
        stack[:len(free)] = free                                          # what lies above the top stays there
        asked, at_most = 0, len(free)
        for pages, a, w in zip(held, lens, wanted):
            more = -(-w // page) - len(pages)
            if -(-w // page) > width:
                w = a
            elif more > 0:
                asked += more
                if asked > at_most:
                    w = a
                else:
                    pages += [free.pop() for _ in range(more)]
            out.append(w)
            positions.append([a + r for r in range(n)])
            slots.append([pages[(a + r) // page] * page + (a + r) % page if a + r < w else -1 for r in range(n)])
        return out, positions, slots

    lens = st["lens"].tolist()
    between, _, _ = resize(lens, st["between"].tolist(), 0)
    lens, positions, slots = resize(between, lens, case["n"])
    return {"table": _ints([pages + [-1] * (width - len(pages)) for pages in held]), "free_pages": _ints(stack), "num_free": _ints([len(free)]),
            "between": _ints(between), "lens": _ints(lens), "positions": _ints(positions), "slots": _ints(slots)}


def _exact_shared(st, case):
    """Sequence by sequence on all of its keys, the prefix's before its own."""
    H, Hkv, d, page = case["H"], case["Hkv"], case["d"], case["page"]
    out = torch.zeros(st["Q"].shape, dtype=torch.float64, device="cuda")
    prefixes, owns, b = _prefix_lengths(case), _own_lengths(case), 0

    def rows(ids, count, name, scale):
        x = st[name].float()[ids].double() if st[scale] is None else st[name].view(torch.uint8)[ids].view(st[name].dtype).double() * st[scale].double()[ids][..., None, None]
        x = x.transpose(0, 1) if name == "Kc" else x.permute(1, 0, 3, 2)
        return x.reshape(Hkv, -1, d)[:, :count]

    for g, count in enumerate(_groups(case)):
        ids = st["prefix_table"][g].long()
        Kp, Vp = rows(ids, prefixes[g], "Kc", "k_scale"), rows(ids, prefixes[g], "Vc", "v_scale")
        for b in range(b, b + count):
            ids = st["block_table"][b].long()
            K, V = torch.cat([Kp, rows(ids, owns[b], "Kc", "k_scale")], 1), torch.cat([Vp, rows(ids, owns[b], "Vc", "v_scale")], 1)
            if K.shape[1]:
                q = st["Q"][b].double().reshape(Hkv, -1, d)
                w = torch.softmax(torch.matmul(q, K.transpose(1, 2).contiguous()) / math.sqrt(d), -1)
                out[b] = torch.matmul(w, V).view(H, -1, d)
        b += 1
    return {"O": out}


def _exact_verify(st, case):
    """Sequence by sequence, draft by draft, from logarithms of the probabilities."""
    B, n = case["B"], case["n"]
    out = torch.full((B, n + 1), -1, dtype=torch.int32)
    accepted, chances, drafted = torch.zeros(B, dtype=torch.int32), torch.zeros((B, n), dtype=torch.float64), _drafted(case)
    tokens, u = st["tokens"].tolist(), st["uniforms"].double().tolist()
    temps = [1.0] * B if st["temperature"] is None else st["temperature"].double().tolist()

    def probabilities(row, t):
        x = row.double()
        if t == 0:
            p = torch.zeros_like(x)
            p[int((x == x.max()).nonzero()[0])] = 1
            return p
        return torch.exp(torch.log_softmax(x / t, 0))

    for b in range(B):
        i, weights = 0, None
        for k in range(drafted[b]):
            x, p = tokens[b][k], probabilities(st["logits_v"][b, k], temps[b])
            if st["logits_d"] is None:
                q = torch.zeros_like(p)
                q[x] = 1
            else:
                q = probabilities(st["logits_d"][b, k], temps[b])
            px, qx = float(p[x]), float(q[x])
            chances[b, k] = 0 if px == 0 else min(1, px / max(qx, 1e-300))
            if weights is None and u[b][k] * qx < px:
                out[b, k] = x
                i += 1
            elif weights is None:
                left = (p - q).clamp(min=0)
                weights = left if float(left.sum()) > 0 else p
        accepted[b] = i
        if weights is None and case["bonus"]:
            weights = probabilities(st["logits_v"][b, i], temps[b])
        if weights is not None:
            c = torch.cumsum(weights, 0)
            out[b, i] = min(int(torch.searchsorted(c, u[b][n] * c[-1], right=True)), case["V"] - 1)
    return {"tokens": out.cuda(), "accepted": accepted.cuda(), "chances": chances.cuda()}
