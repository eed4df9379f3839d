"""Calls of several host threads at once on one stream: each is several launches that hand data over in scratch memory, which threads on
one stream share."""
import sys
import threading

import pytest

import paper_2604_05250_amd as dd
from _paged import ints

pytestmark = pytest.mark.gpu


def _paged(n, lens, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    B, per = len(lens), 64
    Q, Kc, Vc = normal(B, 8, n, 128), normal(B * per, 2, 64, 128), normal(B * per, 2, 128, 64)
    table, held = ints([[b * per + p for p in range(per)] for b in range(B)]), ints(lens)
    assert dd.dd_paged_attention_workspace_bytes(n, B, 8, 2, 128, 64, per, dd.BF16) > 0
    return lambda: dd.dd_paged_attention(Q, Kc, Vc, table, held)


def _dense(seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    Q, K, V = normal(1, 8, 16, 128), normal(1, 8, 2048, 128), normal(1, 8, 2048, 128)
    assert dd.dd_block_attention_cached_workspace_bytes(16, 1, 8, 8, 2048, 128, dd.BF16, dd.BF16) > 0
    return lambda: dd.dd_block_attention_cached(Q, K, V, 512)


def _scores(seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    D, V = (torch.randn((8, 50000), generator=g, device="cuda") for _ in range(2))
    assert dd.dd_verify_scores_workspace_bytes(8, 50000, dd.F32) > 0
    return lambda: torch.stack([x.float() for x in dd.dd_verify_scores(D, V)[:3]])


@pytest.mark.parametrize("stream", ["default", "own"])
def test_threads_on_one_stream(stream):
    import torch
    calls = [_paged(1, [4096], 1), _paged(2, [3000, 700], 2), _dense(3), _scores(4)]
    on = torch.cuda.default_stream() if stream == "default" else torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(on):
        want = [call() for call in calls]
    torch.cuda.synchronize()
    got, start = [[] for _ in calls], threading.Barrier(len(calls))

    def work(call, to):
        start.wait()
        with torch.cuda.stream(on):
            for _ in range(100):
                to.append(call())
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=work, args=a) for a in zip(calls, got)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    torch.cuda.synchronize()
    for k, (w, outs) in enumerate(zip(want, got)):
        assert len(outs) == 100
        wrong = [i for i, o in enumerate(outs) if not torch.equal(o, w)]
        assert not wrong, f"call {k}: {len(wrong)} of {len(outs)} differ"
