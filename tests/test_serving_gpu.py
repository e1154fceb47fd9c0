"""The serving calls together: the example, one captured step, side streams, and a wait that runs out."""
import os
import random
import sys

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import attention, check_attention, u32
from test_prefix_attn_gpu import build, run

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_the_example_runs_and_sharing_does_not_change_lengths_of_sequences():
    import draft_decode
    for share in (True, False):
        answers, cache, n_live = draft_decode.run(samples=6, rounds=5, draft=3, prompt_len=256, vocab=331, share=share)
        lens = cache.lens.tolist()
        assert lens[0] == 255 and lens[1:4] == [0, 0, 0]
        # A sequence holds the prompt and every token of its answer but the last, which was not fed yet.
        assert lens[4:] == [255 + len(a) for a in answers[3:]]
        assert all(0 <= t < 331 for a in answers for t in a)
        used = set()
        for s, n in enumerate(lens):
            used |= set(cache.table[s, :-(-n // 32)].tolist())
        assert used == set(range(n_live))


def test_a_captured_step_replays():
    """extend, write, attend, verify and drop of one step as a CUDA graph: every replay goes on from the state that
    the one before left, as eager calls do."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    B, H, KV, D, V, k = 5, 8, 2, 64, 300, 2

    def state():
        cache, slots, _ = build([200 + i for i in range(B)], [192], [(0, B)], 32, KV, D, torch.bfloat16, seed=9,
                                poison=False)
        big = serve.PagedCache(1, 200, KV, 32, D, cache.n_slots, 40)
        n = cache.pool.shape[1]
        big.pool[:, :n] = cache.pool
        big.table[:, :cache.max_pages] = cache.table
        big.lens.copy_(cache.lens)
        big.refs[:n] = cache.refs
        return big, u32(slots)

    x = [torch.randn((B, h, k + 1, D), generator=gen, device="cuda").bfloat16() for h in (H, KV, KV)]
    q = torch.softmax(torch.randn((B, k, V), generator=gen, device="cuda"), -1)
    draft = torch.randint(0, V, (B, k), generator=gen, device="cuda").int()
    w = torch.randn((H * D, V), generator=gen, device="cuda") / 8
    ua, us = torch.rand((B, k), generator=gen, device="cuda"), torch.rand((B,), generator=gen, device="cuda")
    start, lens, feed = u32([0, B]), u32([192]), u32([k + 1] * B)

    def step(cache, slots, O):
        granted = cache.extend(slots, feed)
        cache.write(0, slots, granted, x[1], x[2])
        cache.attend(0, x[0], O, slots, granted, start, lens)
        p = torch.softmax(O.transpose(1, 2).flatten(2).float() @ w, -1)
        accepted, tokens = serve.verify_draft(p, q, draft, None, ua, us)
        cache.drop(slots, k - accepted)
        return accepted, tokens

    eager, slots = state()
    O = torch.empty_like(x[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    captured, _ = state()
    O2 = torch.empty_like(O)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        warm, ws = state()
        step(warm, ws, O2)          # loads the kernels
        captured.attend(0, x[0], O2, slots, feed, start, lens)   # makes the workspaces of this cache
        captured.extend(slots, u32([0] * B))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(captured, slots, O2)
    for _ in range(4):
        want = step(eager, slots, O)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
        assert torch.equal(O2.view(torch.int16), O.view(torch.int16))
        assert torch.equal(captured.lens, eager.lens) and torch.equal(captured.refs, eager.refs)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("head_dim,n_heads,n_kv_heads", [(64, 8, 2), (96, 6, 3), (128, 32, 8)])
@pytest.mark.parametrize("B,q_len,own", [(64, 1, 900), (40, 3, 2000), (130, 2, 60), (33, 1, 5000)])
def test_pair_items_beside_own_parts_of_all_lengths(head_dim, n_heads, n_kv_heads, B, q_len, own):
    """Several query tiles a kv head, two groups, and own parts from one token to many tiles: every CTA has both kinds
    of work, in unlike amounts for its two streams."""
    r = random.Random(B + head_dim)
    base = [1500, 700]
    groups, shared = [(0, B // 2), (B // 2, B)], [1490, 690]
    lens = [base[0 if i < B // 2 else 1] + r.choice([1, q_len, own // 2, own, r.randint(1, own)]) for i in range(B)]
    n_new = [min(r.randint(0, q_len), lens[i]) for i in range(B)]
    cache, slots, gen = build(lens, shared, groups, 64, n_kv_heads, head_dim, torch.bfloat16, seed=B)
    run(cache, slots, gen, n_heads, q_len, n_new, groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK


def test_attention_on_side_streams():
    """Two caches over the same tensors attend at the same time on two streams, each with a workspace of its own."""
    lens = [1000 + 10 * i for i in range(12)]
    cache, slots, gen = build(lens, [1000], [(0, 12)], 32, 2, 128, torch.bfloat16, seed=4)
    Q = [torch.randn((12, 8, 1, 128), generator=gen, device="cuda").bfloat16() for _ in range(2)]
    s, start, shared = u32(slots), u32([0, 12]), u32([1000])
    want = [attention(cache, 0, x, slots, [1] * 12) for x in Q]
    views = [serve.PagedCache.over(cache.pool, cache.table, cache.lens, cache.refs) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[torch.empty_like(x) for _ in range(5)] for x in Q]
    torch.cuda.synchronize()
    for i in range(5):
        for v, st, x, o in zip(views, streams, Q, outs):
            v.attend(0, x, o[i], s, None, start, shared, stream=st)
    torch.cuda.synchronize()
    for (w, A), o in zip(want, outs):
        for x in o:
            check_attention(x, w, A, 1200, 6.0)


def test_a_wait_that_runs_out_is_reported_and_the_device_stays_usable():
    """As for the other attention calls: an ordinary bounded wait given a limit of 1 ns."""
    lens = [3000 + 50 * i for i in range(40)]
    groups, shared = [(0, 40)], [2900]
    cache, slots, gen = build(lens, shared, groups, 64, 4, 128, torch.bfloat16, seed=2, poison=False)
    run(cache, slots, gen, 16, 1, None, groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK
    Q = torch.randn((40, 16, 1, 128), generator=gen, device="cuda").bfloat16()
    O, s, start, n = torch.empty_like(Q), u32(slots), u32([0, 40]), u32(shared)
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
    run(cache, slots, gen, 16, 1, None, groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK
