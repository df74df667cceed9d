"""Calls on explicit streams without a workspace and without a synchronisation in between: every call's allocations are its stream's
(tests/test_streams_cpu.py says why), so calls on several streams, and fills on the current one, do not meet in one buffer."""
import pytest
import torch

from paper_2506_12355_b200 import api
from test_paged_gpu import make_cache
from test_rope_gpu import make, table

pytestmark = pytest.mark.gpu


def decode_calls():
    """The tile list with its second kernel: partial results in the workspace."""
    lens, D, dt = [900, 2000, 17, 1500] * 6, 128, torch.bfloat16
    kc, vc, tab, _, _ = make_cache(lens, 8, D, 16, dt, "slot", 1, dead=0.0)
    tab, lens = tab.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    for seed in range(3):
        q = torch.randn(24, 32, D, generator=torch.Generator().manual_seed(seed)).to(dt).cuda()
        yield lambda stream, q=q: api.attn_paged_decode(q, kc, vc, tab, lens, 0.09, stream=stream)


def window_calls():
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        q, k, v, d = (torch.randn(1, h, 1500, 64, generator=g).half().cuda() for h in (8, 2, 2, 8))
        o, lse = api.attn_fwd_window(q, k, v, 0.125, 200, 4)
        yield lambda stream, a=(q, k, v, o, lse, d): api.attn_bwd_window(*a, 0.125, 200, 4, stream=stream)


def backward_calls():
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        q, k, v, d = (torch.randn(1, h, 1000, 64, generator=g).half().cuda() for h in (8, 2, 2, 8))
        o, lse = api.attn_fwd_gqa(q, k, v, 0.125, causal=True)
        yield lambda stream, a=(q, k, v, o, lse, d): api.attn_bwd(*a, 0.125, causal=True, stream=stream)


def rope_calls():
    tab = table(700, 128).cuda()
    for seed in range(3):
        q, k, v, qw, kw = make(2, 700, 16, 4, 128, torch.bfloat16, seed)
        grads = [torch.randn_like(t.transpose(1, 2).contiguous()) for t in (q, k, v)]
        yield lambda stream, a=(*grads, q, k, qw, kw, tab): api.attn_qk_norm_rope_bwd(*a, stream=stream)


def splitkv_calls():
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        q, k, v = (torch.randn(1, 4, n, 128, generator=g).bfloat16().cuda() for n in (1, 4096, 4096))
        yield lambda stream, a=(q, k, v): api.attn_fwd_splitkv(*a, 0.09, False, 8, stream=stream)


@pytest.mark.parametrize("make_calls", [decode_calls, window_calls, backward_calls, rope_calls, splitkv_calls])
def test_three_streams_at_once(make_calls):
    calls = list(make_calls())
    want = [call(None) for call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), None]
    for _ in range(10):
        got = []
        for call, stream in zip(calls, streams):
            got.append(call(stream))
            for shift in range(9, 24, 2):      # blocks of many sizes of the current stream's pool, filled at once and dropped
                torch.full((1 << shift,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert api.attn_last_device_status() == 0


def test_a_graph_captured_on_the_calls_stream():
    """The stream argument names the capturing stream: the allocations come from the graph's pool, and replays repeat."""
    call = next(iter(decode_calls()))
    want = call(None)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = call(side)
    for _ in range(3):
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_python_marshalling_gives_the_same(monkeypatch):
    """Without the extension the calls are marshalled in Python: same results, with and without a stream."""
    every = [list(f()) for f in (decode_calls, window_calls, rope_calls)]
    want = [[call(None) for call in calls] for calls in every]
    side = torch.cuda.Stream()
    monkeypatch.setattr(api, "_binding_module", None)
    torch.cuda.synchronize()
    for stream in (None, side):
        for calls, results in zip(every, want):
            for call, result in zip(calls, results):
                got = call(stream)
                torch.cuda.synchronize()
                assert all(torch.equal(x, y) for x, y in zip(got, result))


def test_the_current_stream_stays(monkeypatch):
    """... after a call on another one, after a refused one, and where torch's short cuts to it are missing."""
    q = torch.randn(1, 2, 64, 64, device="cuda").half()
    want = api.attn_fwd_window(q, q, q, 0.125, 8)
    torch.cuda.synchronize()
    outer, inner = torch.cuda.Stream(), torch.cuda.Stream()
    for short_cut in (True, False):
        if not short_cut:
            monkeypatch.setattr(api, "_set_stream", None)
        for current in (torch.cuda.default_stream(), outer):
            with torch.cuda.stream(current):
                for stream in (inner, torch.cuda.default_stream(), torch.cuda.ExternalStream(inner.cuda_stream), current):
                    got = api.attn_fwd_window(q, q, q, 0.125, 8, stream=stream)
                    assert torch.cuda.current_stream() == current
                    stream.synchronize()
                    assert all(torch.equal(a, b) for a, b in zip(got, want))
                    with pytest.raises(ValueError):
                        api.attn_fwd_gqa(q, q[:, :, :, :32], q, 0.125, stream=stream)
                    assert torch.cuda.current_stream() == current
