"""What dd_paged_resize refuses before anything reaches a GPU: through the C ABI (addresses that are never dereferenced) and through the
binding (CPU tensors, which it refuses last of all)."""
import pytest
import torch

import paper_2604_05250_amd as dd

FAKE = 1 << 36
NULL, SHAPE, WORKSPACE, ALIGN = -1, -2, -5, -6


def resize(**kw):
    a = dict(t=FAKE, s=2 * FAKE, f=3 * FAKE, lens=4 * FAKE, new=5 * FAKE, out=6 * FAKE, pos=7 * FAKE, slots=8 * FAKE, n=4, B=3, pages=50, P=16, most=9, ws=9 * FAKE,
             wsn=1 << 30)
    a.update(kw)
    return dd.lib().dd_paged_resize(a["t"], a["s"], a["f"], a["lens"], a["new"], a["out"], a["pos"], a["slots"], a["n"], a["B"], a["pages"], a["P"], a["most"],
                                    a["ws"], a["wsn"], None)


@pytest.mark.parametrize("want,kw", [
    *[(NULL, {name: None}) for name in ("t", "s", "f", "lens", "new", "out", "pos", "slots")],
    (SHAPE, dict(n=-1)), (SHAPE, dict(B=-1)), (SHAPE, dict(pages=0)), (SHAPE, dict(P=8)), (SHAPE, dict(P=48)), (SHAPE, dict(most=0)), (SHAPE, dict(most=1 << 26)),
    (SHAPE, dict(pages=1 << 27)), (SHAPE, dict(n=1 << 30)), (SHAPE, dict(B=1 << 20, n=1 << 11)), (SHAPE, dict(B=1 << 20, most=1 << 11)), (SHAPE, dict(B=1 << 24)),
    (WORKSPACE, dict(B=1 << 16, ws=None)), (WORKSPACE, dict(B=1 << 16, wsn=100)), (WORKSPACE, dict(B=1 << 16, ws=9 * FAKE + 16)),
    *[(ALIGN, {name: 10 * FAKE + 2}) for name in ("t", "s", "f", "lens", "new", "out", "pos", "slots")],
    # what is written overlaps nothing
    (SHAPE, dict(s=FAKE)), (SHAPE, dict(f=FAKE + 3 * 9 * 4 - 4)), (SHAPE, dict(out=FAKE)), (SHAPE, dict(pos=2 * FAKE + 50 * 4 - 4)), (SHAPE, dict(slots=7 * FAKE)),
    (SHAPE, dict(lens=FAKE)), (SHAPE, dict(new=8 * FAKE + 44)), (SHAPE, dict(out=4 * FAKE + 4)), (SHAPE, dict(out=5 * FAKE - 8)), (SHAPE, dict(f=4 * FAKE))])
def test_refused(want, kw):
    assert resize(**kw) == want


def test_no_sequences_do_nothing():
    assert resize(B=0) == 0 and resize(B=0, t=None, lens=None, new=None, out=None, pos=None, slots=None) == 0


def test_workspace_query():
    need = dd.dd_paged_resize_workspace_bytes
    assert need(1, 16, 64, 32) == 0 and need(2048, 64, 16, 128) > 0 and need(0, 1 << 16, 16, 9) > 0
    for bad in ((-1, 16, 64, 32), (1 << 30, 16, 64, 32), (2048, 0, 16, 128), (2048, 64, 17, 128), (2048, 64, 16, 0), (1 << 12, 1 << 20, 16, 1)):
        assert need(*bad) == 0


i32 = torch.int32


def z(*shape, t=i32):
    return torch.zeros(shape, dtype=t)


def bound(page_size=16, n=4, **kw):
    a = dict(block_table=z(3, 9), free_pages=z(50), num_free=z(1), lens=z(3), new_lens=z(3))
    a.update(kw)
    return dd.dd_paged_resize(**a, page_size=page_size, n=n)


@pytest.mark.parametrize("error,match,call", [
    (TypeError, "block_table: a tensor", lambda: bound(block_table=None)), (ValueError, "block_table", lambda: bound(block_table=z(27))),
    (ValueError, "block_table", lambda: bound(block_table=z(3, 9, t=torch.int64))), (ValueError, "free_pages", lambda: bound(free_pages=z(50, t=torch.int64))),
    (ValueError, "num_free: must be int32 with 1", lambda: bound(num_free=z(2))), (ValueError, "lens: must be int32 with 3", lambda: bound(lens=z(2))),
    (ValueError, "new_lens", lambda: bound(new_lens=z(3, t=torch.float32))), (ValueError, "out_lens", lambda: bound(out_lens=z(4))),
    (ValueError, "positions: must be int32 with 12", lambda: bound(positions=z(3, 3))), (ValueError, "slots: must be int32 with 12", lambda: bound(slots=z(3, 4, t=torch.int16))),
    (ValueError, "n: is out of range", lambda: bound(n=-1)), (ValueError, "page_size: is out of range", lambda: bound(page_size=1 << 70)),
    (ValueError, "a size is out of range", lambda: bound(n=1 << 40)), (ValueError, "block_table: must live in GPU memory", lambda: bound())])
def test_binding_refuses(error, match, call):
    with pytest.raises(error, match=match):
        call()


def test_a_float_is_no_size():
    import ctypes
    with pytest.raises(ctypes.ArgumentError):
        bound(n=4.0)
