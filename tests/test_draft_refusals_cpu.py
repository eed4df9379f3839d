"""What dd_verify_draft refuses before anything reaches a GPU: through the C ABI (addresses that are never dereferenced) and through the
binding (CPU tensors, which it refuses last of all)."""
import pytest
import torch

import paper_2604_05250_amd as dd

FAKE = 1 << 30
NULL, SHAPE, DTYPE, WORKSPACE, ALIGN = -1, -2, -3, -5, -6


def verify(**kw):
    a = dict(lv=FAKE, ld=2 * FAKE, tokens=3 * FAKE, count=None, u=4 * FAKE, t=None, ot=5 * FAKE, oa=6 * FAKE, oc=7 * FAKE, B=2, n=3, bonus=1, V=64, dtype=dd.F32,
             ws=8 * FAKE, wsn=1 << 30)
    a.update(kw)
    return dd.lib().dd_verify_draft(a["lv"], a["ld"], a["tokens"], a["count"], a["u"], a["t"], a["ot"], a["oa"], a["oc"], a["B"], a["n"], a["bonus"], a["V"],
                                    a["dtype"], a["ws"], a["wsn"], None)


@pytest.mark.parametrize("want,kw", [
    *[(NULL, {name: None}) for name in ("lv", "tokens", "u", "ot", "oa", "oc")],
    (DTYPE, dict(dtype=dd.FP8_E4M3)), (DTYPE, dict(dtype=9)), (SHAPE, dict(B=-1)), (SHAPE, dict(n=-1)), (SHAPE, dict(V=0)), (SHAPE, dict(n=0, bonus=0)),
    (SHAPE, dict(n=0x7fffffff)), (SHAPE, dict(B=1 << 20, n=1 << 12)), (SHAPE, dict(B=1 << 24)), (ALIGN, dict(V=63)), (ALIGN, dict(V=60, dtype=dd.BF16)),
    (ALIGN, dict(lv=FAKE + 8)), (ALIGN, dict(ld=2 * FAKE + 4)), (ALIGN, dict(tokens=3 * FAKE + 2)), (ALIGN, dict(count=FAKE * 9 + 1)), (ALIGN, dict(u=4 * FAKE + 1)),
    (ALIGN, dict(t=FAKE * 9 + 2)), (ALIGN, dict(ot=5 * FAKE + 2)), (ALIGN, dict(oa=6 * FAKE + 3)), (ALIGN, dict(oc=7 * FAKE + 1)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(wsn=100)), (WORKSPACE, dict(ws=8 * FAKE + 16)),
    # outputs over inputs or each other
    (SHAPE, dict(ot=3 * FAKE)), (SHAPE, dict(ot=3 * FAKE - 28)), (SHAPE, dict(oa=FAKE + 2 * 4 * 64 * 4 - 4)), (SHAPE, dict(oc=2 * FAKE + 2 * 3 * 64 * 4 - 4)),
    (SHAPE, dict(oa=4 * FAKE)), (SHAPE, dict(oc=5 * FAKE + 28)), (SHAPE, dict(oa=9 * FAKE, count=9 * FAKE + 4)), (SHAPE, dict(oa=9 * FAKE, t=9 * FAKE)),
    (SHAPE, dict(oa=7 * FAKE + 20))])
def test_refused(want, kw):
    assert verify(**kw) == want


def test_no_sequences_do_nothing():
    assert verify(B=0) == 0 and verify(B=0, lv=None, tokens=None, u=None, ot=None, oa=None, oc=None) == 0


def test_workspace_query():
    need = dd.dd_verify_draft_workspace_bytes
    assert need(1, 4, 1, 126464, 1, dd.BF16) > need(1, 4, 1, 126464, 0, dd.BF16) > 0 and need(1, 0, 1, 64, 0, dd.F32) > 0
    for bad in ((0, 4, 1, 64, 1, 1), (1, -1, 1, 64, 1, 1), (1, 0, 0, 64, 1, 1), (1, 4, 1, 0, 1, 1), (1, 4, 1, 64, 1, 2), (1 << 24, 4, 1, 64, 1, 1)):
        assert need(*bad) == 0


f32, bf16, i32 = torch.float32, torch.bfloat16, torch.int32


def z(*shape, t=f32):
    return torch.zeros(shape, dtype=t)


def bound(**kw):
    a = dict(logits_v=z(2, 4, 64), logits_d=z(2, 3, 64), tokens=z(2, 3, t=i32), uniforms=z(2, 4))
    a.update(kw)
    return dd.dd_verify_draft(**a)


@pytest.mark.parametrize("error,match,call", [
    (TypeError, "logits_v: a tensor", lambda: bound(logits_v=None)), (TypeError, "tokens: a tensor", lambda: bound(tokens=None)),
    (TypeError, "uniforms: a tensor", lambda: bound(uniforms=None)), (ValueError, "three dimensions", lambda: bound(logits_v=z(8, 64))),
    (ValueError, "three dimensions", lambda: bound(tokens=z(6, t=i32))), (ValueError, "logits_v shape", lambda: bound(logits_v=z(2, 5, 64))),
    (ValueError, "logits_v shape", lambda: bound(logits_v=z(3, 4, 64))), (ValueError, "logits_d shape", lambda: bound(logits_d=z(2, 4, 64))),
    (TypeError, "logits_d: elements", lambda: bound(logits_d=z(2, 3, 64, t=bf16))), (TypeError, "BFloat16 expected", lambda: bound(logits_v=z(2, 4, 64, t=torch.float16), logit_dtype=dd.BF16)),
    (ValueError, "tokens: must have 6", lambda: bound(tokens=z(2, 3, t=torch.int64))), (ValueError, "uniforms: must have 8", lambda: bound(uniforms=z(2, 3))),
    (ValueError, "uniforms: must have 8", lambda: bound(uniforms=z(2, 4, t=torch.float64))), (ValueError, "temperature: must have 2", lambda: bound(temperature=z(1))),
    (ValueError, "n_draft: must have 2", lambda: bound(n_draft=z(2))), (ValueError, "out_tokens: must have 8", lambda: bound(out_tokens=z(2, 3, t=i32))),
    (ValueError, "out_accepted: must have 2", lambda: bound(out_accepted=z(2))), (ValueError, "out_chances: must have 6", lambda: bound(out_chances=z(2, 4))),
    (ValueError, "logits_v: must live in GPU memory", lambda: bound())])
def test_binding_refuses(error, match, call):
    with pytest.raises(error, match=match):
        call()
