"""What dd_paged_attention_shared refuses before anything reaches a GPU: through the C ABI (addresses that are never dereferenced) and
through the binding (CPU tensors, which it refuses last of all)."""
import pytest
import torch

import paper_2604_05250_amd as dd

FAKE = 1 << 36
NULL, SHAPE, DTYPE, WORKSPACE, ALIGN = -1, -2, -3, -5, -6


def attend(**kw):
    a = dict(Q=FAKE, Kc=2 * FAKE, Vc=3 * FAKE, ks=4 * FAKE, vs=5 * FAKE, pt=6 * FAKE, pl=7 * FAKE, gs=8 * FAKE, table=9 * FAKE, lens=10 * FAKE, O=11 * FAKE, n=1,
             B=4, H=8, Hkv=2, d=128, pages=99, P=64, G=2, mp=64, most=4, cache=dd.FP8_E4M3, ws=12 * FAKE, wsn=1 << 30)
    a.update(kw)
    return dd.lib().dd_paged_attention_shared(a["Q"], a["Kc"], a["Vc"], a["ks"], a["vs"], a["pt"], a["pl"], a["gs"], a["table"], a["lens"], a["O"], a["n"], a["B"],
                                              a["H"], a["Hkv"], a["d"], a["pages"], a["P"], a["G"], a["mp"], a["most"], a["cache"], a["ws"], a["wsn"], None)


OUT = 4 * 8 * 128 * 2


@pytest.mark.parametrize("want,kw", [
    *[(NULL, {name: None}) for name in ("Q", "Kc", "Vc", "ks", "vs", "pt", "pl", "gs", "table", "lens", "O")],
    (DTYPE, dict(cache=dd.F32)), (SHAPE, dict(H=7)), (SHAPE, dict(H=0)), (SHAPE, dict(B=0)), (SHAPE, dict(n=-1)), (SHAPE, dict(d=256)), (SHAPE, dict(P=48)),
    (SHAPE, dict(pages=0)), (SHAPE, dict(most=0)), (SHAPE, dict(mp=0)), (SHAPE, dict(G=0)), (SHAPE, dict(G=-1)), (SHAPE, dict(mp=1 << 24)), (SHAPE, dict(most=1 << 24)),
    (SHAPE, dict(n=1 << 28)), (SHAPE, dict(G=1 << 23)), (SHAPE, dict(B=1 << 22)), (ALIGN, dict(Q=FAKE + 8)), (ALIGN, dict(O=11 * FAKE + 8)),
    (ALIGN, dict(vs=5 * FAKE + 1)), (ALIGN, dict(lens=10 * FAKE + 2)), (ALIGN, dict(pt=6 * FAKE + 2)), (ALIGN, dict(pl=7 * FAKE + 1)), (ALIGN, dict(gs=8 * FAKE + 3)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(wsn=64)), (WORKSPACE, dict(ws=12 * FAKE + 16)),
    *[(SHAPE, dict(O=k * FAKE)) for k in range(1, 11)], (SHAPE, dict(O=FAKE + OUT - 16)), (SHAPE, dict(O=8 * FAKE - OUT + 16, gs=8 * FAKE)),
    (SHAPE, dict(O=9 * FAKE + 4 * 4 * 4 - 16)), (SHAPE, dict(O=2 * FAKE + 99 * 2 * 64 * 128 - 16))])
def test_refused(want, kw):
    assert attend(**kw) == want


def test_launches_have_fewer_than_2_32_threads():
    # (a workspace that would do: what is refused is the size)
    big = dict(H=2, Hkv=2, pages=99, wsn=1 << 62)
    assert attend(B=1 << 20, **big) == SHAPE and attend(B=(1 << 20) - 4, G=4, **dict(big, ws=None)) == WORKSPACE
    assert attend(B=1, n=1 << 26, **big) == SHAPE and attend(B=1, G=1 << 21, **big) == SHAPE


def test_without_queries_does_nothing():
    assert attend(n=0) == 0 and attend(n=0, Q=None, O=None) == 0


def test_workspace_query():
    need = dd.dd_paged_attention_shared_workspace_bytes
    ok = (1, 4, 8, 2, 128, 64, 2, 64, 4, 2)
    assert need(*ok) > 0
    for i, bad in ((0, 0), (1, 0), (2, 7), (3, 0), (4, 96), (5, 65), (6, 0), (7, 0), (8, 0), (9, 0), (7, 1 << 24), (6, 1 << 23)):
        assert need(*(bad if k == i else v for k, v in enumerate(ok))) == 0


f32, bf16, u8, i32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32


def z(*shape, t=bf16):
    return torch.zeros(shape, dtype=t)


def bound(**kw):
    a = dict(Q=z(3, 4, 5, 64), Kc=z(9, 2, 16, 64, t=u8), Vc=z(9, 2, 64, 16, t=u8), prefix_table=z(2, 7, t=i32), prefix_lens=z(2, t=i32), group_starts=z(3, t=i32),
             block_table=z(3, 4, t=i32), kv_lens=z(3, t=i32), k_scale=z(9, 2, t=f32), v_scale=z(9, 2, t=f32))
    a.update(kw)
    return dd.dd_paged_attention_shared(**a)


@pytest.mark.parametrize("error,match,call", [
    (TypeError, "Q: a tensor", lambda: bound(Q=None)), (TypeError, "group_starts: a tensor", lambda: bound(group_starts=None)),
    (ValueError, "shapes must be Kc", lambda: bound(Vc=z(9, 2, 16, 64, t=u8))), (ValueError, "block_table", lambda: bound(block_table=z(12, t=i32))),
    (ValueError, "prefix_table", lambda: bound(prefix_table=z(14, t=i32))), (ValueError, "prefix_table", lambda: bound(prefix_table=z(2, 7, t=torch.int64))),
    (ValueError, "Q shape", lambda: bound(Q=z(2, 4, 5, 64))), (ValueError, "Q shape", lambda: bound(Q=z(3, 4, 5, 128))), (TypeError, "Q: elements", lambda: bound(Q=z(3, 4, 5, 64, t=f32))),
    (TypeError, "Q: BFloat16", lambda: bound(Q=z(3, 4, 5, 64, t=torch.float16))), (ValueError, "kv_lens: must be int32 with 3", lambda: bound(kv_lens=z(2, t=i32))),
    (ValueError, "prefix_lens: must be int32 with 2", lambda: bound(prefix_lens=z(3, t=i32))), (ValueError, "group_starts: must be int32 with 3", lambda: bound(group_starts=z(2, t=i32))),
    (ValueError, "group_starts: must be int32 with 3", lambda: bound(group_starts=z(3, t=f32))), (ValueError, "O: too small", lambda: bound(O=z(3, 4, 5, 63))),
    (ValueError, "k_scale: too small", lambda: bound(k_scale=z(17, t=f32))), (TypeError, "v_scale: float32", lambda: bound(v_scale=z(9, 2))),
    (ValueError, "Q: must live in GPU memory", lambda: bound())])
def test_binding_refuses(error, match, call):
    with pytest.raises(error, match=match):
        call()
