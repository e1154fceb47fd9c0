"""The calls on caches in 8 or 4 bits together: the example, a captured step, work of all kinds at once, a wait that runs
out."""
import os
import random
import sys

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from quant_helpers import Twin, build, check_attention, stored
from serve_helpers import attention, u32
from test_quant_attn_gpu import run

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("share", [True, False])
def test_the_example(bits, share):
    import draft_decode
    answers, cache, n_live = draft_decode.run(samples=6, rounds=5, draft=3, prompt_len=256, vocab=331, share=share, bits=bits)
    lens = cache.lens.tolist()
    assert cache.bits == bits and lens[0] == 255 and lens[1:4] == [0, 0, 0]
    assert lens[4:] == [255 + len(a) for a in answers[3:]]
    assert all(0 <= t < 331 for a in answers for t in a)
    used = set()
    for s, n in enumerate(lens):
        used |= set(cache.table[s, :-(-n // 32)].tolist())
    assert used == set(range(n_live))


@pytest.mark.parametrize("bits", [4, 8])
def test_steps_of_several_layers(bits):
    """A prompt, forks, rounds of drafts that are written, attended to and partly dropped, in three layers; then a
    compaction and a dense read of everything."""
    page, kv, heads, dim, layers, B = 32, 2, 8, 128, 3, 5
    dtype = torch.bfloat16
    c = serve.PagedCache(layers, 80, kv, page, dim, B + 1, 12, dtype, bits=bits)
    c.pool.random_(0, 256)
    gen = torch.Generator(device="cuda").manual_seed(bits)
    said = [[torch.empty((2, kv, 0, dim), dtype=torch.float64, device="cuda") for _ in range(B + 1)] for _ in range(layers)]
    twin = Twin(c, torch.zeros((2 * layers, 80, kv, page, dim), dtype=torch.float64, device="cuda"))

    def grow(slots, n):
        granted = c.extend(u32(slots), u32(n))
        assert granted.tolist() == n
        for layer in range(layers):
            x = torch.randn((2, len(slots), kv, max(n), dim), generator=gen, device="cuda").to(dtype)
            c.write(layer, u32(slots), granted, x[0], x[1])
            for i, s in enumerate(slots):
                said[layer][s] = torch.cat([said[layer][s], stored(x[:, i, :, :n[i]], bits)], 2)
        return granted

    def mirror():
        for layer in range(layers):
            for s in range(B + 1):
                at = torch.arange(said[layer][s].shape[2], device="cuda")
                page_of, off = c.table[s].long()[at // page], at % page
                for k in range(2):
                    twin.pool[2 * layer + k, page_of, :, off] = said[layer][s][k].transpose(0, 1)

    grow([0], [137])
    slots = list(range(1, B + 1))
    c.fork(u32([0] * B), u32(slots))
    for layer in range(layers):
        for s in slots:
            said[layer][s] = said[layer][0]
    r = random.Random(bits)
    start, shared = u32([0, B]), u32([137])
    for _ in range(4):
        n = [r.randint(1, 5) for _ in slots]
        granted = grow(slots, n)
        mirror()
        for layer in range(layers):
            Q = torch.randn((B, heads, 5, dim), generator=gen, device="cuda").to(dtype)
            O = torch.empty_like(Q)
            c.attend(layer, Q, O, u32(slots), granted, start, shared)
            want, A = attention(twin, layer, Q, slots, n)
            check_attention(O, want, A, 200, 6.0)
        gone = [r.randint(0, x) for x in n]
        c.drop(u32(slots), u32(gone))
        for layer in range(layers):
            for s, g in zip(slots, gone):
                said[layer][s] = said[layer][s][:, :, :said[layer][s].shape[2] - g]
    c.drop(u32([2, 4]), u32([1 << 20, 40]))
    for layer in range(layers):
        said[layer][2], said[layer][4] = said[layer][2][:, :, :0], said[layer][4][:, :, :-40]
    c.compact()
    rows = max(x.shape[2] for x in said[0])
    for layer in range(layers):
        out = torch.empty((2, B + 1, kv, rows, dim), dtype=dtype, device="cuda")
        c.read(layer, out[0], out[1], u32(list(range(B + 1))))
        for s in range(B + 1):
            n = said[layer][s].shape[2]
            assert torch.equal(out[:, s, :, :n].double(), said[layer][s]) and not out[:, s, :, n:].any()
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
def test_a_captured_step_replays(bits):
    """extend, write, attend, drop and read of one step as a CUDA graph goes on from the state that the replay before
    left, as eager calls do."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    B, H, KV, D, k = 5, 8, 2, 64, 2
    x = [torch.randn((B, h, k + 1, D), generator=gen, device="cuda").bfloat16() for h in (H, KV, KV)]
    start, shared, feed, gone = u32([0, B]), u32([192]), u32([k + 1] * B), u32([0, 1, 2, 1, 0])

    def state():
        cache, _, slots, _ = build(bits, [200 + i for i in range(B)], 32, KV, D, torch.bfloat16, 9, [(0, B)], [192])
        big = serve.PagedCache(1, 200, KV, 32, D, cache.n_slots, 40, bits=bits)
        n = cache.n_pages
        big.pool[:, :n] = cache.pool
        big.table[:, :cache.max_pages] = cache.table
        big.lens.copy_(cache.lens)
        big.refs[:n] = cache.refs
        return big, u32(slots)

    def step(cache, slots, O, out):
        granted = cache.extend(slots, feed)
        cache.write(0, slots, granted, x[1], x[2])
        cache.attend(0, x[0], O, slots, granted, start, shared)
        cache.drop(slots, gone)
        cache.read(0, out[0], out[1], slots)

    eager, slots = state()
    captured, _ = state()
    O, out = torch.empty_like(x[0]), torch.empty((2, B, KV, 230, D), dtype=torch.bfloat16, device="cuda")
    O2, out2 = torch.empty_like(O), torch.empty_like(out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm, ws = state()
        step(warm, ws, O2, out2)
        captured.attend(0, x[0], O2, slots, feed, start, shared)   # makes the workspaces of this cache
        captured.extend(slots, u32([0] * B))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured, slots, O2, out2)
    for _ in range(4):
        step(eager, slots, O, out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O2.view(torch.int16), O.view(torch.int16)) and torch.equal(out2, out)
        assert torch.equal(captured.lens, eager.lens) and torch.equal(captured.refs, eager.refs)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("head_dim,n_heads,n_kv_heads", [(64, 8, 2), (96, 6, 3), (128, 32, 8)])
@pytest.mark.parametrize("B,q_len,own", [(64, 1, 900), (40, 3, 2000), (130, 2, 60), (33, 1, 5000)])
def test_prefixes_beside_own_parts_of_all_lengths(bits, head_dim, n_heads, n_kv_heads, B, q_len, own):
    """Several row tiles a kv head, two groups, and own parts from one token to many steps: every CTA has both kinds of
    work, segments that end inside its run and rows that join parts of several CTAs."""
    r = random.Random(B + head_dim)
    base = [1500, 700]
    groups, shared = [(0, B // 2), (B // 2, B)], [1490, 690]
    lens = [base[0 if i < B // 2 else 1] + r.choice([1, q_len, own // 2, own, r.randint(1, own)]) for i in range(B)]
    n_new = [min(r.randint(0, q_len), lens[i]) for i in range(B)]
    cache, twin, slots, gen = build(bits, lens, 64, n_kv_heads, head_dim, torch.bfloat16, B, groups, shared)
    run(cache, twin, slots, gen, n_heads, q_len, n_new, groups, shared)
    run(cache, twin, slots, gen, n_heads, q_len, n_new)
    assert wise.wise_get_status() == wise.WISE_OK


def test_the_largest_batch():
    """1024 requests, 256 groups."""
    B = 1024
    lens = [40 + i % 7 for i in range(B)]
    groups, shared = [(4 * g, 4 * g + 4) for g in range(256)], [32 + g % 3 for g in range(256)]
    cache, twin, slots, gen = build(4, lens, 16, 1, 64, torch.bfloat16, 5, groups, shared)
    run(cache, twin, slots, gen, 4, 1, None, groups, shared)
    run(cache, twin, slots, gen, 4, 1)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("grouped", [True, False])
def test_a_wait_that_runs_out_is_reported_and_the_device_stays_usable(bits, grouped):
    """An ordinary bounded wait given a limit of 1 ns (the hardware holds a wait for some microseconds before the limit is
    looked at, so there has to be one that lasts: that for the buffer of the queries two segments on)."""
    B = 40 if grouped else 160
    lens = [9000 + 50 * i for i in range(B)] if grouped else [2000 + i for i in range(B)]
    groups, shared = ([(0, B)], [8900]) if grouped else (None, None)
    cache, twin, slots, gen = build(bits, lens, 64, 4, 128, torch.bfloat16, 2, groups or (), shared or ())
    run(cache, twin, slots, gen, 16, 1, None, groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK
    Q = torch.randn((B, 16, 1, 128), generator=gen, device="cuda").bfloat16()
    O, s = torch.empty_like(Q), u32(slots)
    start, n = (u32([0, B]), u32(shared)) if grouped else (None, None)
    status = wise.WISE_OK
    wise.wise_set_wait_limit_ns(1)
    try:
        for _ in range(3):
            cache.attend(0, Q, O, s, None, start, n)
            status = wise.wise_get_status()
            if status != wise.WISE_OK:
                break
    finally:
        wise.wise_set_wait_limit_ns(0)
    assert status == wise.WISE_ERR_TIMEOUT
    assert wise.wise_get_status() == wise.WISE_OK
    run(cache, twin, slots, gen, 16, 1, None, groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK
