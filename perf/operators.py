"""The operators between a projection and the attention calls, and the attention over a paged cache, on the sizes that
their callers use.

A case is one of three kinds:
  rotate  dd_qk_norm_rope: per-head norms of queries and keys and the rotation by position, from a fused projection's rows
  append  dd_paged_cache_append: keys (normed and rotated on the way) and values into pages of bf16 or e4m3
  attend  dd_paged_attention: a block's queries over the pages of their sequences
With `own` false, run() computes them in plain torch operations; with `own` true, it calls this package.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
EPS = 1e-6


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one token of one sequence: nothing but latency
        _rotate("rotate_bf16_token", B=1, H=32, Hkv=8, n=1, d=128, dtype="bf16", base=511),
        # the checkable size: fp32, odd length, pairs side by side, half of the head dims rotated
        _rotate("rotate_f32_n333", B=1, H=4, Hkv=2, n=333, d=64, dtype="f32", interleaved=True, rot=32),
        # the active blocks of a throughput batch, far into long sequences
        _rotate("rotate_bf16_block_b16", B=16, H=32, Hkv=8, n=64, d=128, dtype="bf16", base=130000),
        # the verifier's pass over a throughput batch: the largest stream of bytes
        _rotate("rotate_bf16_b16_n2048", B=16, H=32, Hkv=8, n=2048, d=128, dtype="bf16"),
        # one token for each sequence of a serving batch
        _append("append_fp8_token_b16", B=16, Hkv=8, n=1, N=2048, d=128, page=64, cache="fp8"),
        # short blocks of an odd serving batch at unaligned positions
        _append("append_fp8_block_b11", B=11, Hkv=8, n=16, N=1237, d=128, page=64, cache="fp8"),
        # the prompt of one long sequence into bf16 pages, no head norm
        _append("append_bf16_n4096", B=1, Hkv=32, n=4096, N=4096, d=128, page=16, cache="bf16", norm=False),
        # the prompts of a throughput batch
        _append("append_fp8_b16_n2048", B=16, Hkv=8, n=2048, N=2048, d=128, page=64, cache="fp8"),
        # one token of one sequence over a short context
        _attend("attend_fp8_token_n512", B=1, H=32, Hkv=8, n=1, N=512, d=128, page=64, cache="fp8"),
        # one token for each sequence of a serving batch over long contexts: the cache is read once, little else happens
        _attend("attend_fp8_token_b16_n4096", B=16, H=32, Hkv=8, n=1, N=4096, d=128, page=64, cache="fp8"),
        # the drafter's call of a batch of eight on bf16 pages
        _attend("attend_bf16_block_b8_n1024", B=8, H=32, Hkv=32, n=64, N=1024, d=128, page=16, cache="bf16"),
        # the drafter's call of a throughput batch with grouped heads: compute bound
        _attend("attend_fp8_block_b16_n2048", B=16, H=32, Hkv=8, n=64, N=2048, d=128, page=64, cache="fp8"),
    ]


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "attend", "attend"])
    d = 64 if rng.random() < 0.2 else 128
    H, Hkv = rng.choice([(4, 2), (28, 4), (32, 32)] if d == 64 else [(32, 32), (32, 8), (28, 4), (16, 16)])
    B = _log_int(rng, 1, 16)
    if kind == "rotate":
        n = _log_int(rng, 1, 4096)
        while B * n * (H + Hkv) > 16 * 2048 * 40:             # no more than the largest listed call
            n = max(1, n // 2)
        return _rotate(None, B=B, H=H, Hkv=Hkv, n=n, d=d, dtype=rng.choice(["bf16", "bf16", "f32"]), base=_log_int(rng, 1, 200000),
                       interleaved=rng.random() < 0.3, rot=rng.choice([d, d, d // 2]), norm=rng.random() < 0.8)
    page, cache = rng.choice([16, 32, 64, 64, 128]), rng.choice(["fp8", "fp8", "bf16"])
    N = _log_int(rng, 64, 4096)
    if kind == "append":
        n = min(N, _log_int(rng, 1, 2048))
        while B * n * Hkv > 16 * 2048 * 8:
            n = max(1, n // 2)
        return _append(None, B=B, Hkv=Hkv, n=n, N=N, d=d, page=page, cache=cache, norm=rng.random() < 0.7,
                       interleaved=rng.random() < 0.3, rot=rng.choice([d, d, d // 2]))
    n = rng.choice([1, 1, 8, 16, 24, 32, 48, 64])
    while B * H * n * N * d > 16 * 32 * 64 * 2048 * 128:
        N = N // 2
    return _attend(None, B=B, H=H, Hkv=Hkv, n=n, N=N, d=d, page=page, cache=cache)


def _rotate(name, B, H, Hkv, n, d, dtype, base=0, interleaved=False, rot=None, norm=True):
    return _named(name, dict(kind="rotate", B=B, H=H, Hkv=Hkv, n=n, d=d, dtype=dtype, base=base, interleaved=interleaved,
                             rot=rot or d, norm=norm))


def _append(name, B, Hkv, n, N, d, page, cache, norm=True, interleaved=False, rot=None):
    return _named(name, dict(kind="append", B=B, Hkv=Hkv, n=n, N=N, d=d, page=page, cache=cache, norm=norm,
                             interleaved=interleaved, rot=rot or d))


def _attend(name, B, H, Hkv, n, N, d, page, cache):
    return _named(name, dict(kind="attend", B=B, H=H, Hkv=Hkv, n=n, N=N, d=d, page=page, cache=cache))


def _named(name, case):
    return case if name is None else dict(case, name=name)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _lengths(case):
    """Sequence lengths of a ragged batch: the first is N, the others down to three quarters of it."""
    N, least = case["N"], case.get("n", 1) if case["kind"] == "append" else 1
    return [max(least, N - (b * 97) % (N // 4 + 1)) for b in range(case["B"])]


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": dict(case)}
    B, n, d = case["B"], case["n"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    if case["kind"] != "attend":
        half = case["rot"] // 2
        st["inv_freq"] = (500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()
    if case["kind"] == "rotate":
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        H, Hkv = case["H"], case["Hkv"]
        rows = (1.5 * normal(B, n, (H + 2 * Hkv) * d)).to(dt)          # a fused projection's output: q, k, v
        st["Q"] = rows[..., :H * d].view(B, n, H, d).transpose(1, 2)
        st["K"] = rows[..., H * d:(H + Hkv) * d].view(B, n, Hkv, d).transpose(1, 2)
        st["q_weight"] = (1 + 0.1 * normal(d)).to(dt) if case["norm"] else None
        st["k_weight"] = (1 + 0.1 * normal(d)).to(dt) if case["norm"] else None
        first = torch.randint(0, case["base"] + 1, (B, 1), generator=g, device="cuda")
        st["positions"] = (first + torch.arange(n, device="cuda")).to(torch.int32)
        st["Qo"] = torch.empty((B, H, n, d), dtype=dt, device="cuda")
        st["Ko"] = torch.empty((B, Hkv, n, d), dtype=dt, device="cuda")
        return st
    Hkv, page, N = case["Hkv"], case["page"], case["N"]
    per = -(-N // page)
    pages = B * per + 3                                                # a pool with a few pages that no sequence holds
    st["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    st["table"] = torch.randperm(pages, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)
    kshape, vshape = (pages, Hkv, page, d), (pages, Hkv, d, page)
    if case["cache"] == "fp8":
        st["Kc"] = (70 * normal(*kshape)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        st["Vc"] = (70 * normal(*vshape)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        st["k_scale"] = torch.exp2(torch.randint(-7, -5, (pages, Hkv), generator=g, device="cuda").float())
        st["v_scale"] = torch.exp2(torch.randint(-7, -5, (pages, Hkv), generator=g, device="cuda").float())
    else:
        st["Kc"], st["Vc"] = normal(*kshape).bfloat16(), normal(*vshape).bfloat16()
        st["k_scale"] = st["v_scale"] = None
    if case["kind"] == "append":
        rows = (1.5 * normal(B, n, 2 * Hkv * d)).bfloat16()            # the key and value part of a projection's output
        st["K"] = rows[..., :Hkv * d].view(B, n, Hkv, d).transpose(1, 2)
        st["V"] = rows[..., Hkv * d:].view(B, n, Hkv, d).transpose(1, 2)
        st["k_weight"] = (1 + 0.1 * normal(d)).bfloat16() if case["norm"] else None
        st["starts"] = st["lens"] - n
        return st
    st["Q"] = (1.5 * normal(B, case["H"], n, d)).bfloat16()
    st["O"] = torch.empty_like(st["Q"])
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if own:
        return _run_own(st, case)
    if case["kind"] == "rotate":
        turn = _turns(st["positions"], st["inv_freq"])
        return {name: _rotated(_normed(st[src].float(), st[w]), turn, case["interleaved"]).to(st[src].dtype)
                for name, src, w in (("Q", "Q", "q_weight"), ("K", "K", "k_weight"))}
    if case["kind"] == "append":
        return _append_plain(st, case)
    return {"O": _attend_plain(st, case)}


def _run_own(st, case):
    import paper_2604_05250_amd as dd
    if case["kind"] == "rotate":
        Qo, Ko = dd.dd_qk_norm_rope(st["Q"], st["K"], q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, inv_freq=st["inv_freq"],
                                    positions=st["positions"], interleaved=case["interleaved"], Qo=st["Qo"], Ko=st["Ko"])
        return {"Q": Qo, "K": Ko}
    if case["kind"] == "append":
        dd.dd_paged_cache_append(st["Kc"], st["Vc"], st["K"], st["V"], st["table"], st["starts"], st["starts"], k_scale=st["k_scale"],
                                 v_scale=st["v_scale"], k_weight=st["k_weight"], eps=EPS, inv_freq=st["inv_freq"],
                                 interleaved=case["interleaved"])
        return _cache_of(st)
    return {"O": dd.dd_paged_attention(st["Q"], st["Kc"], st["Vc"], st["table"], st["lens"], k_scale=st["k_scale"],
                                       v_scale=st["v_scale"], O=st["O"])}


def _cache_of(st):
    got = {"Kc": st["Kc"], "Vc": st["Vc"]}
    if st["k_scale"] is not None:
        got["k_scale"], got["v_scale"] = st["k_scale"], st["v_scale"]
    return got


# ---------------------------------------------------------------- the plain forms
def _normed(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _turns(positions, inv_freq):
    """cos and sin of every position's angles, [B, 1, n, rot/2]; the angles in 64 bits, as positions go far."""
    a = (positions.double().unsqueeze(-1) * inv_freq.double()).unsqueeze(1)
    return torch.cos(a).float(), torch.sin(a).float()


def _rotated(x, turn, interleaved):
    c, s = turn
    half = c.shape[-1]
    rot, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        u, v = rot[..., 0::2], rot[..., 1::2]
        return torch.cat([torch.stack([u * c - v * s, v * c + u * s], -1).flatten(-2), rest], -1)
    u, v = rot[..., :half], rot[..., half:]
    return torch.cat([u * c - v * s, v * c + u * s, rest], -1)


def _append_plain(st, case):
    """The pages that a call touches are taken out of the cache, rebuilt and put back."""
    B, n, page = case["B"], case["n"], case["page"]
    starts = st["starts"].long()
    K = _rotated(_normed(st["K"].float(), st["k_weight"]),
                 _turns(starts.unsqueeze(1) + torch.arange(n, device="cuda"), st["inv_freq"]), case["interleaved"])
    touched = (n + page - 2) // page + 1                                # pages that n rows can touch, wherever they begin
    pos = (starts // page * page).unsqueeze(1) + torch.arange(touched * page, device="cuda")
    row = pos - starts.unsqueeze(1)
    written = ((row >= 0) & (row < n)).view(B, touched, page)
    kept = (row < 0).view(B, touched, page)
    index = (starts // page).unsqueeze(1) + torch.arange(touched, device="cuda")
    ids = st["table"].long().gather(1, index.clamp(max=st["table"].shape[1] - 1))
    real = written.any(-1) & (index < st["table"].shape[1])             # a touched page holds a row
    ids, written, kept = ids[real], written[real], kept[real]
    at = row.clamp(0, n - 1)
    batch = torch.arange(B, device="cuda").unsqueeze(1)
    new_k = K.transpose(1, 2)[batch, at].view(B, touched, page, -1, case["d"])[real].transpose(1, 2)
    new_v = st["V"].float().transpose(1, 2)[batch, at].view(B, touched, page, -1, case["d"])[real].permute(0, 2, 3, 1)
    _put(st["Kc"], st["k_scale"], ids, new_k, written[:, None, :, None], kept[:, None, :, None])
    _put(st["Vc"], st["v_scale"], ids, new_v, written[:, None, None, :], kept[:, None, None, :])
    return _cache_of(st)


def _put(cache, scale, ids, new, written, kept):
    if scale is None:
        cache[ids] = torch.where(written, new.to(cache.dtype), cache[ids])
        return
    codes = cache.view(torch.uint8)
    old = codes[ids]
    amax = (new.abs() * written).amax((-2, -1))
    m, e = torch.frexp(amax)                                            # amax = m 2^e, 1/2 <= m < 1; 448 = 0.875 2^9
    want = torch.where(amax > 0, (e - 9 + (m > 0.875)).clamp(min=-126), -126)
    s = torch.ldexp(torch.ones_like(amax), want)
    had = scale[ids]
    s = torch.where(kept.flatten(1).any(-1, keepdim=True), torch.maximum(s, had), s)
    grown = old.view(cache.dtype).float() * (had / s)[..., None, None]
    codes[ids] = torch.where(written, (new / s[..., None, None]).to(cache.dtype).view(torch.uint8),
                             torch.where(kept, grown.to(cache.dtype).view(torch.uint8), old))
    scale[ids] = s


def _attend_plain(st, case):
    B, H, Hkv, n, d = (case[k] for k in ("B", "H", "Hkv", "n", "d"))
    ids = st["table"].long()
    K, V = _held(st["Kc"], st["k_scale"], ids), _held(st["Vc"], st["v_scale"], ids)
    K = K.permute(0, 2, 4, 1, 3).reshape(B * Hkv, d, -1)
    V = V.permute(0, 2, 1, 4, 3).reshape(B * Hkv, -1, d)
    Q = st["Q"].float().view(B * Hkv, H // Hkv * n, d)
    S = torch.bmm(Q, K) * (1.0 / math.sqrt(d))
    keys = torch.arange(S.shape[-1], device="cuda")
    hidden = (keys >= st["lens"].unsqueeze(1)).repeat_interleave(Hkv, 0).unsqueeze(1)
    S = S.masked_fill(hidden, -math.inf)
    P = torch.exp(S - S.amax(-1, keepdim=True))
    return (torch.bmm(P, V) / P.sum(-1, keepdim=True)).view(B, H, n, d).to(st["Q"].dtype)


def _held(cache, scale, ids):
    """The values of the sequences' pages, [B, pages, Hkv, page, d] or [B, pages, Hkv, d, page]."""
    if scale is None:
        return cache[ids].float()
    return cache.view(torch.uint8)[ids].view(cache.dtype).float() * scale[ids][..., None, None]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    B, n, d = case["B"], case["n"], case["d"]
    if case["kind"] == "rotate":
        el = 2 if case["dtype"] == "bf16" else 4
        x = B * n * (case["H"] + case["Hkv"]) * d
        return {"bytes": 2 * x * el + 4 * B * n, "flops": (4 if case["norm"] else 0) * x + 3 * x * case["rot"] / d}
    el, Hkv, page = 1 if case["cache"] == "fp8" else 2, case["Hkv"], case["page"]
    lens = _lengths(case)
    scales = (0 if case["cache"] == "bf16" else 8 * Hkv)
    if case["kind"] == "append":
        x = B * n * Hkv * d
        touched = sum((t - 1) // page - (t - n) // page + 1 for t in lens)
        return {"bytes": 2 * x * 2 + 2 * x * el + touched * (scales + 4),
                "flops": x * ((4 if case["norm"] else 0) + 3 * case["rot"] / d + (4 if el == 1 else 0))}
    keys, pages = sum(lens), sum(-(-t // page) for t in lens)
    return {"bytes": 2 * 2 * B * case["H"] * n * d + 2 * keys * Hkv * d * el + pages * (scales + 4),
            "flops": 4 * case["H"] * n * d * keys}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rotate":
        return {name: _exact_rows(st[name], st[w], st["positions"], st["inv_freq"], case["interleaved"])
                for name, w in (("Q", "q_weight"), ("K", "k_weight"))}
    return _exact_append(st, case) if case["kind"] == "append" else {"O": _exact_attend(st, case)}


def _exact_rows(x, w, positions, inv_freq, interleaved):
    """Rows as complex numbers, one for each pair of dims, times e^(i angle)."""
    y = x.to(torch.float64, copy=True)
    if w is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + EPS) * w.double()
    half = inv_freq.shape[0]
    k = torch.arange(half, device=x.device)
    i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + half)
    angle = positions.double()[:, None, :, None] * inv_freq.double()
    z = torch.complex(y[..., i], y[..., j]) * torch.polar(torch.ones_like(angle), angle)
    y[..., i], y[..., j] = z.real, z.imag
    return y


def _exact_append(st, case):
    """Sequence by sequence, page by page."""
    n, page, starts = case["n"], case["page"], st["starts"].tolist()
    where = st["starts"].double().unsqueeze(1) + torch.arange(n, device="cuda")
    K = _exact_rows(st["K"], st["k_weight"], where, st["inv_freq"], case["interleaved"])
    V = st["V"].double()
    table = st["table"].tolist()
    fp8 = st["k_scale"] is not None
    out = {}
    for name, rows, scale in (("Kc", K, "k_scale"), ("Vc", V, "v_scale")):
        cache = st[name].float() if fp8 else st[name].double()          # the values that codes stand for, per unit of scale
        if name == "Vc":
            cache = cache.transpose(-1, -2)
        cache = cache.clone()
        s = st[scale].double() if fp8 else None
        for b, t in enumerate(starts):
            for p in range(t // page, (t + n - 1) // page + 1):
                lo, hi = max(t, p * page), min(t + n, (p + 1) * page)
                id_ = table[b][p]
                new = rows[b, :, lo - t:hi - t]
                at, end = lo - p * page, hi - p * page
                if fp8:
                    a = new.abs().amax((-2, -1))
                    need = torch.exp2(torch.ceil(torch.log2(a / E4M3_MAX)).clamp(min=-126))
                    need = torch.where(a > E4M3_MAX * need, 2 * need, torch.where(a <= E4M3_MAX * need / 2, need / 2, need)).clamp(min=2.0 ** -126)
                    if at:
                        need = torch.maximum(need, s[id_])
                        cache[id_, :, :at] = _nearest_e4m3(cache[id_, :, :at].double() * (s[id_] / need)[:, None, None]).float()
                    s[id_] = need
                    new = _nearest_e4m3(new / need[:, None, None])
                cache[id_, :, at:end] = new.to(cache.dtype)
        out[name] = cache.transpose(-1, -2).contiguous() if name == "Vc" else cache
        if fp8:
            out[scale] = s
    return out


def _nearest_e4m3(x):
    """Three mantissa bits down to 2^-6, steps of 2^-9 below; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_attend(st, case):
    """Sequence by sequence, on its own keys only."""
    H, Hkv, d, page = case["H"], case["Hkv"], case["d"], case["page"]
    out = torch.empty(st["Q"].shape, dtype=torch.float64, device="cuda")
    for b, t in enumerate(_lengths(case)):
        ids = st["table"][b, :-(-t // page)].long()
        K, V = (c.float()[ids].double() for c in (st["Kc"], st["Vc"]))
        if st["k_scale"] is not None:
            K, V = K * st["k_scale"].double()[ids, :, None, None], V * st["v_scale"].double()[ids, :, None, None]
        K = K.transpose(0, 1).reshape(Hkv, -1, d)[:, :t].repeat_interleave(H // Hkv, 0)
        V = V.permute(1, 0, 3, 2).reshape(Hkv, -1, d)[:, :t].repeat_interleave(H // Hkv, 0)
        w = torch.softmax(torch.matmul(st["Q"][b].double(), K.transpose(1, 2).contiguous()) / math.sqrt(d), -1)
        out[b] = torch.matmul(w, V)
    return out
