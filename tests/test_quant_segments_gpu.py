"""Attention over caches in 8 or 4 bits where a CTA goes through much more than its rings hold: segments of many pages,
many segments, references that move late; against the definition in fp64."""
import random

import pytest
import torch

from paper_2609_27373_gb300 import wise
from quant_helpers import Twin, build, check_attention, stored
from serve_helpers import attention, u32
from test_quant_attn_gpu import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("page,head_dim,n_heads", [(16, 64, 8), (32, 96, 4), (128, 128, 8), (16, 128, 72)])
def test_segments_of_many_pages(bits, page, head_dim, n_heads):
    """Segments that pass 32 pages several times, with more and with at most 16 query rows; ids out of range far behind
    their first page."""
    lens = [3000 - 7 * i for i in range(40)]
    cache, twin, slots, gen = build(bits, lens, page, 4, head_dim, torch.bfloat16, page + head_dim)
    run(cache, twin, slots, gen, n_heads, 1)
    bad = [5, 17, 39]
    for i, at in zip(bad, (lens[5] - 1, 2300, 1100)):
        cache.table[slots[i], at // page] = cache.n_pages + i
    Q = torch.randn((40, n_heads, 1, head_dim), generator=gen, device="cuda").to(torch.bfloat16)
    O = torch.full_like(Q, float("nan"))
    cache.attend(0, Q, O, u32(slots))
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    want, A = attention(twin, 0, Q, [-1 if i in bad else s for i, s in enumerate(slots)], [1] * 40)
    check_attention(O, want, A, 3000, float(twin.pool.abs().max()))
    assert not O[bad].any()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("q_len,n_heads,grouped", [(1, 6, False), (4, 6, True), (5, 30, False)])
def test_many_short_items(bits, q_len, n_heads, grouped):
    """More than 16 segments a CTA, most of one step, empty ones and rows without new tokens among them."""
    B, r = 700, random.Random(bits + q_len)
    least = 210 if grouped else 0
    lens = [least + r.choice([0, 1, 5, 128, 129, 200, 256, 257, r.randint(0, 300)]) for _ in range(B)]
    groups, shared = ([(0, 90), (90, 640)], [200, 70]) if grouped else ((), ())
    n_new = [min(r.randint(0, q_len), n) for n in lens]
    cache, twin, slots, gen = build(bits, lens, 16, 6, 64, torch.float16, q_len, groups, shared)
    slots[7] = slots[300] = -1
    run(cache, twin, slots, gen, n_heads, q_len, n_new, groups or None, shared or None)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,flip", [(40, False), (40, True), (3, False), (64, False)])
def test_references_that_move_in_every_step(bits, rows, flip):
    """Logits that grow by more than a numerator's range from step to step, in the last one too, where rows of the same
    request see different keys; rows of the same item whose references move and rows whose do not."""
    n, D = 1500, 128
    cache, twin, slots, gen = build(bits, [n, n], 64, 1, D, torch.bfloat16, 41)
    size = torch.linspace(0.05, 30.0, n, device="cuda")
    size = size.flip(0) if flip else size
    K = (torch.ones((2, 1, n, D), device="cuda") * size[:, None]).to(torch.bfloat16)
    V = torch.randn((2, 1, n, D), generator=gen, device="cuda").to(torch.bfloat16)
    cache.write(0, u32(slots), u32([n, n]), K, V)
    for s, at in zip(slots, range(2)):
        for p in range(-(-n // 64)):
            page, m = int(cache.table[s, p]), min(64, n - 64 * p)
            twin.pool[0, page, :, :m] = stored(K[at, :, 64 * p:64 * p + m], bits)
            twin.pool[1, page, :, :m] = stored(V[at, :, 64 * p:64 * p + m], bits)
    q_len = 1 if rows == 3 else 4
    heads = rows // q_len
    way = torch.tensor([1.0, -1.0, 0.02, 0.0], device="cuda")[torch.arange(heads, device="cuda") % 4]
    Q = (torch.ones((2, heads, q_len, D), device="cuda") * way[:, None, None]).to(torch.bfloat16)
    O = torch.full_like(Q, float("nan"))
    cache.attend(0, Q, O, u32(slots))
    want, A = attention(twin, 0, Q, slots, [q_len] * 2)
    check_attention(O, want, A, n, float(V.abs().max()) * 1.1)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits,page,head_dim,n_heads", [(8, 32, 96, 4), (4, 32, 96, 4), (8, 64, 128, 4), (4, 16, 64, 4),
                                                        (8, 32, 96, 80), (4, 64, 128, 80)])
def test_repeats_with_cold_caches(bits, page, head_dim, n_heads):
    """Loads that end out of order: pages come from memory in every second call, and all calls give the same bits."""
    lens = [3000 - 7 * i for i in range(40)]
    cache, twin, slots, gen = build(bits, lens, page, 4, head_dim, torch.bfloat16, page + head_dim)
    Q, first = run(cache, twin, slots, gen, n_heads, 1)
    flush, s, outs = torch.empty(300 << 20, dtype=torch.uint8, device="cuda"), u32(slots), []
    for i in range(100):
        if i % 2:
            flush.fill_(i)
        outs.append(torch.full_like(Q, float("nan")))
        cache.attend(0, Q, outs[-1], s)
    assert all(torch.equal(O, first) for O in outs)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_heads", [5, 20])
def test_other_calls_leave_no_trace(bits, n_heads):
    """The same bits whatever ran before: items of few rows that end inside a step after calls with more rows and large
    logits of either sign."""
    lens = [257 + i % 128 for i in range(200)]
    cache, twin, slots, gen = build(bits, lens, 64, 1, 64, torch.bfloat16, 3)
    other, _, theirs, _ = build(bits, [2000] * 200, 64, 1, 64, torch.bfloat16, 4)
    Q, first = run(cache, twin, slots, gen, n_heads, 1)
    s, t, X = u32(slots), u32(theirs), torch.empty((200, 16 if n_heads == 5 else 64, 1, 64), dtype=torch.bfloat16, device="cuda")
    for i in range(12):
        X.copy_(torch.randn(X.shape, generator=gen, device="cuda") * (0.0, 30.0, 300.0)[i % 3])
        other.attend(0, X, torch.empty_like(X), t)
        O = torch.full_like(Q, float("nan"))
        cache.attend(0, Q, O, s)
        assert torch.equal(O, first)
    assert wise.wise_get_status() == wise.WISE_OK
