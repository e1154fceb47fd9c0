"""Graphs captured from a cache's calls, replayed after larger calls on the same cache."""
import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import u32

pytestmark = pytest.mark.gpu


def test_a_small_step_replays_after_larger_calls():
    """A step of two requests is captured, then calls of 64 need larger workspaces: replays still give what eager
    calls give, and write nothing outside the memory that the cache holds."""
    page, KV, D, H, B = 16, 2, 64, 8, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    pool = torch.randn((2, 900, KV, page, D), generator=gen, device="cuda").bfloat16()
    lens = [100 + s for s in range(B)]

    def filled():
        cache = serve.PagedCache(1, 900, KV, page, D, B, 14)
        cache.extend(u32(list(range(B))), u32(lens))
        cache.pool.copy_(pool)
        return cache

    x = [torch.randn((B, h, 1, D), generator=gen, device="cuda").bfloat16() for h in (H, KV, KV)]
    every, ones, zeros = u32(list(range(B))), u32([1] * B), u32([0] * B)
    outs = {}

    def step(cache, n):
        O = outs.setdefault((id(cache), n), torch.zeros((n, H, 1, D), dtype=torch.bfloat16, device="cuda"))
        granted = cache.extend(every[:n], ones[:n])
        cache.write(0, every[:n], granted, x[1][:n], x[2][:n])
        cache.attend(0, x[0][:n], O, every[:n], granted)
        return O

    def read_all(cache):
        O = outs.setdefault((id(cache), "all"), torch.zeros((B, H, 1, D), dtype=torch.bfloat16, device="cuda"))
        cache.extend(every, zeros)
        cache.attend(0, x[0], O, every)
        return O

    eager, graphed = filled(), filled()
    # Its list workspace is to grow as well.
    graphed._kv_ws, graphed._kv_n, graphed._workspaces = None, -1, []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        warm = filled()
        step(warm, 2)
        graphed.attend(0, x[0][:2], torch.empty((2, H, 1, D), dtype=torch.bfloat16, device="cuda"), every[:2])
        graphed.extend(every[:2], zeros[:2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        O2 = step(graphed, 2)
    captured = list(graphed._workspaces)
    assert len(captured) == 2
    read_all(graphed)
    assert len(graphed._workspaces) >= 3
    # Memory that comes after: what the allocator would have had back is handed out here.
    later = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")
             for ws in captured for n in [ws.numel()] * 8]
    with torch.cuda.stream(side):
        later += [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")
                  for ws in captured for n in [ws.numel()] * 8]
    torch.cuda.synchronize()
    assert {t.data_ptr() for t in captured} <= {t.data_ptr() for t in graphed._workspaces}
    for _ in range(3):
        graph.replay()
        want = step(eager, 2)
        torch.cuda.synchronize()
        assert torch.equal(O2.view(torch.int16), want.view(torch.int16))
        assert torch.equal(read_all(graphed).view(torch.int16), read_all(eager).view(torch.int16))
        assert torch.equal(graphed.lens, eager.lens) and torch.equal(graphed.refs, eager.refs)
    assert all(bool((t == 0x5A).all()) for t in later)
    assert wise.wise_get_status() == wise.WISE_OK
