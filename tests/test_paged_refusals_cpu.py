"""What the calls around a paged cache refuse before anything reaches a GPU: through the C ABI (addresses that are never dereferenced)
and through the binding (CPU tensors, which it refuses last of all)."""
import pytest
import torch

import paper_2604_05250_amd as dd

FAKE = 1 << 20
NULL, SHAPE, DTYPE, WORKSPACE, ALIGN = -1, -2, -3, -5, -6


def rope(**kw):
    a = dict(Q=FAKE, q=(4 * 9 * 64, 9 * 64, 64), K=2 * FAKE, k=(2 * 9 * 64, 9 * 64, 64), qw=None, kw=None, eps=1e-6, freq=FAKE, rot=64, inter=0,
             pos=FAKE, Qo=3 * FAKE, Ko=4 * FAKE, B=2, H=4, Hkv=2, n=9, d=64, dtype=dd.F32)
    a.update(kw)
    return dd.lib().dd_qk_norm_rope(a["Q"], *a["q"], a["K"], *a["k"], a["qw"], a["kw"], a["eps"], a["freq"], a["rot"], a["inter"], a["pos"], a["Qo"],
                                    a["Ko"], a["B"], a["H"], a["Hkv"], a["n"], a["d"], a["dtype"], None)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(Q=None)), (NULL, dict(Qo=None)), (NULL, dict(K=None)), (NULL, dict(Ko=None)), (NULL, dict(freq=None)),
    (DTYPE, dict(dtype=dd.FP8_E4M3)), (DTYPE, dict(dtype=7)), (SHAPE, dict(d=96)), (SHAPE, dict(B=0)), (SHAPE, dict(H=0)), (SHAPE, dict(Hkv=0)),
    (SHAPE, dict(n=-1)), (SHAPE, dict(B=1 << 16, n=1 << 15)), (SHAPE, dict(rot=-16)), (SHAPE, dict(rot=8)), (SHAPE, dict(rot=80)),
    (SHAPE, dict(qw=FAKE, eps=0.0)), (SHAPE, dict(kw=FAKE, eps=float("nan"))), (SHAPE, dict(qw=FAKE, eps=float("inf"))), (SHAPE, dict(qw=FAKE, eps=-1.0)),
    (SHAPE, dict(q=(-64, 64, 64))), (SHAPE, dict(k=(1 << 41, 64, 64))), (ALIGN, dict(q=(4 * 9 * 64, 9 * 64, 65))), (ALIGN, dict(k=(1, 64, 64))),
    (ALIGN, dict(Q=FAKE + 4)), (ALIGN, dict(Ko=4 * FAKE + 8)), (ALIGN, dict(qw=FAKE + 4)), (ALIGN, dict(kw=FAKE + 4)), (ALIGN, dict(pos=FAKE + 2)),
    (ALIGN, dict(freq=FAKE + 2)),
    # outputs over inputs or each other, but for a dense input of their own
    (SHAPE, dict(Qo=FAKE + 256)), (SHAPE, dict(Qo=2 * FAKE)), (SHAPE, dict(Ko=FAKE)), (SHAPE, dict(Ko=3 * FAKE)), (SHAPE, dict(Ko=3 * FAKE + 2 * 4 * 9 * 64 * 4 - 16)),
    (SHAPE, dict(Qo=FAKE, q=(4 * 9 * 64, 64, 4 * 64)))])
def test_rope_is_refused(want, kw):
    assert rope(**kw) == want


def test_rope_without_tokens_does_nothing():
    assert rope(n=0) == 0 and rope(n=0, Q=None, Qo=None, K=None, Ko=None) == 0


def append(**kw):
    a = dict(Kc=FAKE, Vc=2 * FAKE, ks=FAKE, vs=FAKE, K=3 * FAKE, k=(2 * 5 * 64, 5 * 64, 64), V=4 * FAKE, v=(2 * 5 * 64, 5 * 64, 64), table=FAKE, starts=FAKE,
             lens=None, count=None, w=None, eps=1e-6, freq=FAKE, rot=64, inter=0, n=5, B=2, Hkv=2, d=64, pages=9, P=16, most=4, row=dd.BF16, cache=dd.FP8_E4M3)
    a.update(kw)
    return dd.lib().dd_paged_cache_append(a["Kc"], a["Vc"], a["ks"], a["vs"], a["K"], *a["k"], a["V"], *a["v"], a["table"], a["starts"], a["lens"], a["count"],
                                          a["w"], a["eps"], a["freq"], a["rot"], a["inter"], a["n"], a["B"], a["Hkv"], a["d"], a["pages"], a["P"], a["most"],
                                          a["row"], a["cache"], None)


@pytest.mark.parametrize("want,kw", [
    *[(NULL, {name: None}) for name in ("Kc", "Vc", "ks", "vs", "K", "V", "table", "starts", "freq")],
    (DTYPE, dict(cache=dd.F32)), (DTYPE, dict(row=dd.FP8_E4M3)), (SHAPE, dict(d=32)), (SHAPE, dict(n=-1)), (SHAPE, dict(B=0)), (SHAPE, dict(Hkv=0)),
    (SHAPE, dict(pages=0)), (SHAPE, dict(most=0)), (SHAPE, dict(P=8)), (SHAPE, dict(P=48)), (SHAPE, dict(P=256)), (SHAPE, dict(most=1 << 28)),
    (SHAPE, dict(pages=1 << 30)), (SHAPE, dict(rot=24)), (SHAPE, dict(w=FAKE, eps=0.0)), (SHAPE, dict(v=(-8, 64, 64))),
    (SHAPE, dict(n=1 << 30, k=(0, 0, 64), v=(0, 0, 64), B=64)), (ALIGN, dict(k=(4, 64, 64))), (ALIGN, dict(v=(64, 64, 68))), (ALIGN, dict(Kc=FAKE + 8)),
    (ALIGN, dict(V=FAKE + 2)), (ALIGN, dict(table=FAKE + 1)), (ALIGN, dict(lens=FAKE + 2)), (ALIGN, dict(count=FAKE + 3)), (ALIGN, dict(ks=FAKE + 2)),
    (ALIGN, dict(w=FAKE + 2))])
def test_append_is_refused(want, kw):
    assert append(**kw) == want


@pytest.mark.parametrize("kw", [
    dict(Vc=FAKE), dict(Vc=FAKE + 9 * 2 * 16 * 64 - 16), dict(K=FAKE), dict(V=FAKE + 9 * 2 * 16 * 64 - 16), dict(K=2 * FAKE + 64), dict(V=2 * FAKE),
    dict(K=2 * FAKE - (2 * 2 * 5 * 64 * 2 - 16))])
def test_append_refuses_rows_in_the_cache(kw):
    assert append(**kw) == SHAPE


def test_launches_have_fewer_than_2_32_threads():
    big = 1 << 29
    assert rope(B=1, n=big, d=128, rot=128, K=None, Ko=None, H=1, q=(0, 0, 128), Qo=1 << 50) == SHAPE
    assert append(B=1, n=1 << 27, d=128, Hkv=1, k=(0, 0, 128), v=(0, 0, 128)) == SHAPE
    assert append(B=1 << 22, n=1, d=128, P=128, Hkv=1, k=(128, 0, 0), v=(128, 0, 0)) == SHAPE
    assert attend(B=1 << 21, H=8, Hkv=8) == SHAPE and attend(B=1, H=1, Hkv=1, n=1 << 29) == SHAPE
    assert dd.dd_paged_attention_workspace_bytes(1, 1 << 21, 8, 8, 128, 64, 64, dd.BF16) == 0


@pytest.mark.parametrize("kw", [
    dict(O=1 << 40), dict(O=(1 << 40) + 8 * 128 * 2 - 16), dict(O=1 << 30), dict(O=(1 << 30) + 99 * 2 * 64 * 128 - 16), dict(O=(1 << 31) - (8 * 128 * 2 - 16))])
def test_attention_refuses_an_output_over_its_inputs(kw):
    assert attend(Q=1 << 40, Kc=1 << 30, Vc=1 << 31, ws=1 << 45, wsn=1 << 40, **kw) == SHAPE


def test_append_without_rows_does_nothing():
    assert append(n=0) == 0 and append(n=0, K=None, V=None) == 0


def attend(**kw):
    a = dict(Q=FAKE, Kc=FAKE, Vc=FAKE, ks=FAKE, vs=FAKE, table=FAKE, lens=FAKE, O=2 * FAKE, n=1, B=1, H=8, Hkv=2, d=128, pages=99, P=64, most=64,
             cache=dd.FP8_E4M3, ws=None, wsn=0)
    a.update(kw)
    return dd.lib().dd_paged_attention(a["Q"], a["Kc"], a["Vc"], a["ks"], a["vs"], a["table"], a["lens"], a["O"], a["n"], a["B"], a["H"], a["Hkv"], a["d"],
                                       a["pages"], a["P"], a["most"], a["cache"], a["ws"], a["wsn"], None)


@pytest.mark.parametrize("want,kw", [
    *[(NULL, {name: None}) for name in ("Q", "Kc", "Vc", "ks", "vs", "table", "lens", "O")],
    (DTYPE, dict(cache=dd.F32)), (SHAPE, dict(H=7)), (SHAPE, dict(H=0)), (SHAPE, dict(B=0)), (SHAPE, dict(n=-1)), (SHAPE, dict(d=256)), (SHAPE, dict(P=0)),
    (SHAPE, dict(pages=0)), (SHAPE, dict(most=0)), (SHAPE, dict(n=1 << 29)), (ALIGN, dict(Q=FAKE + 8)), (ALIGN, dict(O=FAKE + 8)), (ALIGN, dict(vs=FAKE + 1)),
    (ALIGN, dict(lens=FAKE + 2)), (WORKSPACE, dict()), (WORKSPACE, dict(ws=FAKE)), (WORKSPACE, dict(ws=FAKE + 16, wsn=1 << 30))])
def test_attention_is_refused(want, kw):
    assert attend(**kw) == want


def test_attention_without_queries_does_nothing():
    assert attend(n=0) == 0 and attend(n=0, Q=None, O=None) == 0


def test_workspace_query():
    need = dd.dd_paged_attention_workspace_bytes
    assert need(1, 1, 8, 2, 128, 64, 64, dd.FP8_E4M3) > 0 and need(1, 1, 8, 2, 128, 64, 1, dd.FP8_E4M3) == 0
    for bad in ((0, 1, 8, 2, 128, 64, 64, 2), (1, 0, 8, 2, 128, 64, 64, 2), (1, 1, 7, 2, 128, 64, 64, 2), (1, 1, 8, 2, 96, 64, 64, 2), (1, 1, 8, 2, 128, 65, 64, 2),
                (1, 1, 8, 2, 128, 64, 0, 2), (1, 1, 8, 2, 128, 64, 64, 0), (1, 1, 8, 2, 128, 64, 1 << 27, 2), (1 << 28, 1, 8, 2, 128, 64, 64, 2)):
        assert need(*bad) == 0


# ---------------------------------------------------------------- the binding
f32, bf16, u8, i32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32


def z(*shape, t=bf16):
    return torch.zeros(shape, dtype=t)


def rows(**kw):
    a = dict(Q=z(2, 4, 5, 64), K=z(2, 2, 5, 64), inv_freq=z(32, t=f32), positions=z(2, 5, t=i32))
    a.update(kw)
    return dd.dd_qk_norm_rope(**a)


def pages(**kw):
    a = dict(Kc=z(9, 2, 16, 64, t=u8), Vc=z(9, 2, 64, 16, t=u8), K=z(2, 2, 5, 64), V=z(2, 2, 5, 64), block_table=z(2, 4, t=i32), starts=z(2, t=i32),
             k_scale=z(9, 2, t=f32), v_scale=z(9, 2, t=f32))
    a.update(kw)
    return dd.dd_paged_cache_append(**a)


def attention(**kw):
    a = dict(Q=z(2, 4, 5, 64), Kc=z(9, 2, 16, 64, t=u8), Vc=z(9, 2, 64, 16, t=u8), block_table=z(2, 4, t=i32), kv_lens=z(2, t=i32), k_scale=z(9, 2, t=f32),
             v_scale=z(9, 2, t=f32))
    a.update(kw)
    return dd.dd_paged_attention(**a)


@pytest.mark.parametrize("error,match,call", [
    (TypeError, "Q: a tensor", lambda: rows(Q=None)), (ValueError, "four dimensions", lambda: rows(Q=z(2, 5, 64))), (ValueError, "K shape", lambda: rows(K=z(2, 2, 6, 64))),
    (ValueError, "Ko and k_weight", lambda: rows(K=None, k_weight=z(64))), (TypeError, "K: elements", lambda: rows(K=z(2, 2, 5, 64, t=f32))),
    (TypeError, "q_weight: elements", lambda: rows(q_weight=z(64, t=f32))), (ValueError, "k_weight: must have 64", lambda: rows(k_weight=z(65))),
    (TypeError, "inv_freq: float32", lambda: rows(inv_freq=z(32))), (ValueError, "inv_freq: has more", lambda: rows(inv_freq=z(33, t=f32))),
    (ValueError, "positions: must be int32 with 10", lambda: rows(positions=z(5, t=i32))), (ValueError, "positions", lambda: rows(positions=z(2, 5, t=torch.int64))),
    (ValueError, "Qo: too small", lambda: rows(Qo=z(2, 4, 5, 63))), (TypeError, "Ko: elements", lambda: rows(Ko=z(2, 2, 5, 64, t=f32))),
    (ValueError, "Q: the last dimension", lambda: rows(Q=z(2, 4, 64, 5).transpose(2, 3), K=None)), (TypeError, "unsupported tensor dtype", lambda: rows(Q=z(2, 4, 5, 64, t=torch.float64), K=None)),
    (ValueError, "Q: must live in GPU memory", lambda: rows()), (ValueError, "Q: must live in GPU memory", lambda: rows(Q=z(2, 5, 4, 64).transpose(1, 2))),
    (ValueError, "shapes must be Kc", lambda: pages(Vc=z(9, 2, 16, 64, t=u8))), (ValueError, "block_table", lambda: pages(block_table=z(8, t=i32))),
    (ValueError, "block_table", lambda: pages(block_table=z(2, 4, t=torch.int64))), (TypeError, "Vc: elements", lambda: pages(Vc=z(9, 2, 64, 16))),
    (ValueError, "k_scale: too small", lambda: pages(k_scale=z(17, t=f32))), (TypeError, "v_scale: float32", lambda: pages(v_scale=z(9, 2))),
    (ValueError, "K and V shapes", lambda: pages(K=z(1, 2, 5, 64), V=z(1, 2, 5, 64))), (ValueError, "K and V shapes", lambda: pages(V=z(2, 2, 4, 64))),
    (TypeError, "V: elements", lambda: pages(V=z(2, 2, 5, 64, t=f32))), (ValueError, "starts", lambda: pages(starts=z(3, t=i32))), (ValueError, "kv_lens", lambda: pages(kv_lens=z(1, t=i32))),
    (ValueError, "n_rows", lambda: pages(n_rows=z(2, t=f32))), (ValueError, "Kc: must live", lambda: pages()),
    (ValueError, "Q shape", lambda: attention(Q=z(3, 4, 5, 64))), (ValueError, "Q shape", lambda: attention(Q=z(2, 4, 5, 128))), (TypeError, "Q: elements", lambda: attention(Q=z(2, 4, 5, 64, t=f32))),
    (ValueError, "kv_lens", lambda: attention(kv_lens=z(1, t=i32))), (ValueError, "O: too small", lambda: attention(O=z(2, 4, 5, 63))), (ValueError, "Q: must live", lambda: attention())])
def test_binding_refuses(error, match, call):
    with pytest.raises(error, match=match):
        call()
