"""A fixed workspace belongs to the thread that has set it: what other threads call meanwhile has its own scratch memory."""
import threading

import pytest

import paper_2604_05250_amd as dd

pytestmark = pytest.mark.gpu


def _in_thread(f):
    box = []

    def work():
        try:
            box.append(f())
        except BaseException as e:                           # handed on to the test
            box.append(e)
    t = threading.Thread(target=work)
    t.start()
    t.join()
    if isinstance(box[0], BaseException):
        raise box[0]
    return box[0]


def test_other_threads_do_not_use_it():
    import torch
    q, kv = torch.randn((1, 8, 16, 128), device="cuda").bfloat16(), torch.randn((1, 8, 2048, 128), device="cuda").bfloat16()
    need = dd.dd_block_attention_cached_workspace_bytes(16, 1, 8, 8, 2048, 128, dd.BF16, dd.BF16)
    assert need > 0
    call = lambda: dd.dd_block_attention_cached(q, kv, kv, 0)
    want = call()
    ws = torch.full((need,), 0xAB, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with dd.fixed_workspace(ws):
        got = _in_thread(call)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and bool((ws == 0xAB).all())
        assert torch.equal(call(), want) and not bool((ws == 0xAB).all())
    # one that is too small is refused in its own thread only
    with dd.fixed_workspace(ws[:256]):
        assert torch.equal(_in_thread(call), want)
        with pytest.raises(RuntimeError, match="fixed workspace"):
            call()
    assert torch.equal(call(), want)


def test_peaks_are_a_threads_own():
    import torch
    q, kv = torch.randn((1, 8, 16, 128), device="cuda").bfloat16(), torch.randn((1, 8, 2048, 128), device="cuda").bfloat16()
    need = dd.dd_block_attention_cached_workspace_bytes(16, 1, 8, 8, 2048, 128, dd.BF16, dd.BF16)
    dd.reset_workspace_peak()
    _in_thread(lambda: dd.dd_block_attention_cached(q, kv, kv, 0))
    assert dd.workspace_peak() == 0
    dd.dd_block_attention_cached(q, kv, kv, 0)
    _in_thread(dd.reset_workspace_peak)
    assert dd.workspace_peak() == need
