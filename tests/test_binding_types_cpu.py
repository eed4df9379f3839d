"""Tensors whose elements have the width of a call's type but are numbers of another kind (fp16 beside bf16, e5m2 beside e4m3) would be
read as what they are not; integers of that width are taken as the bits.  On CPU tensors, which the binding refuses last of all."""
import pytest
import torch

import paper_2604_05250_amd as dd

bf16, f16, f32, u8, i32, e5m2 = torch.bfloat16, torch.float16, torch.float32, torch.uint8, torch.int32, torch.float8_e5m2
fnuz = torch.float8_e4m3fnuz


def z(*shape, t=bf16):
    return torch.zeros(shape, dtype=t)


def rows(**kw):
    a = dict(Q=z(2, 4, 5, 64), K=z(2, 2, 5, 64), inv_freq=z(32, t=f32))
    return dd.dd_qk_norm_rope(**dict(a, **kw))


def append(**kw):
    a = dict(Kc=z(9, 2, 16, 64, t=u8), Vc=z(9, 2, 64, 16, t=u8), K=z(2, 2, 5, 64), V=z(2, 2, 5, 64), block_table=z(2, 4, t=i32), starts=z(2, t=i32),
             k_scale=z(9, 2, t=f32), v_scale=z(9, 2, t=f32))
    return dd.dd_paged_cache_append(**dict(a, **kw))


def attention(**kw):
    a = dict(Q=z(2, 4, 5, 64), Kc=z(9, 2, 16, 64, t=u8), Vc=z(9, 2, 64, 16, t=u8), block_table=z(2, 4, t=i32), kv_lens=z(2, t=i32), k_scale=z(9, 2, t=f32),
             v_scale=z(9, 2, t=f32))
    return dd.dd_paged_attention(**dict(a, **kw))


def dense(**kw):
    a = dict(Q=z(1, 2, 64, 64), K=z(1, 2, 64, 64), V=z(1, 2, 64, 64))
    return dd.dd_bidir_attention(**dict(a, **kw))


@pytest.mark.parametrize("call", [
    lambda: rows(K=z(2, 2, 5, 64, t=f16)), lambda: rows(q_weight=z(64, t=f16)), lambda: rows(k_weight=z(64, t=f16)), lambda: rows(Qo=z(2, 4, 5, 64, t=f16)),
    lambda: rows(Ko=z(2, 2, 5, 64, t=f16)), lambda: rows(Q=z(2, 4, 5, 64, t=f16), K=None, dtype=dd.BF16),
    lambda: append(V=z(2, 2, 5, 64, t=f16)), lambda: append(k_weight=z(64, t=f16)), lambda: append(Vc=z(9, 2, 64, 16, t=e5m2)),
    lambda: append(Kc=z(9, 2, 16, 64, t=fnuz), cache_dtype=dd.FP8_E4M3), lambda: attention(Q=z(2, 4, 5, 64, t=f16)), lambda: attention(O=z(2, 4, 5, 64, t=f16)),
    lambda: attention(Vc=z(9, 2, 64, 16, t=e5m2)), lambda: dense(K=z(1, 2, 64, 64, t=f16)), lambda: dense(V=z(1, 2, 64, 64, t=f16), v_dtype=dd.BF16)])
def test_other_numbers_of_the_same_width_are_refused(call):
    with pytest.raises(TypeError, match="expected, has (Half|Float8)"):
        call()


@pytest.mark.parametrize("call", [
    lambda: rows(Q=z(2, 4, 5, 64, t=torch.int16), K=z(2, 2, 5, 64), q_weight=z(64, t=torch.int16)), lambda: rows(Q=z(2, 4, 5, 64, t=i32), K=None, dtype=dd.F32),
    lambda: append(Kc=z(9, 2, 16, 64, t=torch.float8_e4m3fn)), lambda: append(Kc=z(9, 2, 16, 64), Vc=z(9, 2, 64, 16, t=torch.int16)),
    lambda: attention(Q=z(2, 4, 5, 64, t=torch.int16)), lambda: dense(K=z(1, 2, 64, 64, t=torch.int16))])
def test_bits_are_taken(call):
    with pytest.raises(ValueError, match="must live in GPU memory"):
        call()
