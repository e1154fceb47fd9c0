"""Attention over caches in 8 or 4 bits against its definition in fp64 on the values that the cache stands for."""
import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from quant_helpers import build, check_attention
from serve_helpers import attention, u32

pytestmark = pytest.mark.gpu


def run(cache, twin, slots, gen, n_heads, q_len, n_new=None, groups=None, shared=None, scale=0.0, layer=0, strength=1.5,
        n_keys=None):
    B = len(slots)
    Q = (torch.randn((B, n_heads, q_len, cache.head_dim), generator=gen, device="cuda") * strength).to(cache.dtype)
    O = torch.full_like(Q, float("nan"))
    start = None if groups is None else u32([groups[0][0]] + [b for _, b in groups])
    cache.attend(layer, Q, O, u32(slots), None if n_new is None else u32(n_new), start,
                 None if shared is None else u32(shared), scale)
    new = n_new if n_new is not None else [q_len] * B
    want, A = attention(twin, layer, Q, slots, new, scale)
    lens = cache.lens.tolist()
    check_attention(O, want, A, max([lens[s] for s in slots if s >= 0] + [0]), float(twin.pool.abs().max()))
    return Q, O


CACHES = [(64, 4, 4, 16, torch.bfloat16), (64, 8, 2, 64, torch.float16), (96, 5, 5, 32, torch.float16),
          (96, 24, 4, 128, torch.bfloat16), (128, 32, 8, 64, torch.bfloat16), (128, 3, 3, 128, torch.float16),
          (128, 16, 1, 16, torch.bfloat16), (96, 6, 2, 16, torch.bfloat16), (64, 2, 1, 128, torch.float16)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("head_dim,n_heads,n_kv_heads,page,dtype", CACHES)
@pytest.mark.parametrize("q_len", [1, 3])
def test_lengths(bits, head_dim, n_heads, n_kv_heads, page, dtype, q_len):
    """Sequences of one token up to some tiles, ends inside tiles and pages, an empty one."""
    lens = [q_len, 17, 127, 128, 129, 256, 300, 0, 1000]
    n_new = [min(n, 1 + i % q_len) for i, n in enumerate(lens)]
    cache, twin, slots, gen = build(bits, lens, page, n_kv_heads, head_dim, dtype, seed=head_dim + page + q_len)
    run(cache, twin, slots, gen, n_heads, q_len, n_new)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("head_dim,n_heads,n_kv_heads,page,dtype", CACHES)
@pytest.mark.parametrize("q_len", [1, 3])
def test_shared_prefix(bits, head_dim, n_heads, n_kv_heads, page, dtype, q_len):
    lens = [700 + 3, 700 + 130, 701 + q_len, 700 + 1, 1200, 700 + 64]
    n_new = [1 + i % q_len for i in range(len(lens))]
    groups, shared = [(0, 6)], [700]
    cache, twin, slots, gen = build(bits, lens, page, n_kv_heads, head_dim, dtype, head_dim + page, groups, shared)
    run(cache, twin, slots, gen, n_heads, q_len, n_new, groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
def test_many_requests_of_two_groups(bits):
    """Groups of more rows than a tile has, requests outside of them, unused and repeated slots."""
    lens = [640 + 7 * i % 200 for i in range(70)] + [400 + i for i in range(33)] + [5, 2000, 130]
    groups, shared = [(0, 70), (70, 103)], [600, 390]
    cache, twin, slots, gen = build(bits, lens, 64, 2, 128, torch.bfloat16, 11, groups, shared)
    slots[3] = slots[80] = -1
    slots[105] = slots[104]
    run(cache, twin, slots, gen, 8, 1, None, groups, shared)
    run(cache, twin, slots, gen, 8, 2, [1 + i % 2 for i in range(106)], groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_heads,n_kv_heads,q_len", [(16, 1, 8), (33, 1, 2), (64, 1, 2), (1, 1, 65), (10, 2, 13), (7, 7, 17)])
def test_rows(bits, n_heads, n_kv_heads, q_len):
    """Up to 128 query rows a kv head, odd numbers among them."""
    lens = [q_len, 500, 129, 1]
    n_new = [q_len, q_len // 2 + 1, q_len, 1]
    cache, twin, slots, gen = build(bits, lens, 32, n_kv_heads, 128, torch.float16, 5)
    n_new = [min(a, b) for a, b in zip(n_new, lens)]
    run(cache, twin, slots, gen, n_heads, q_len, n_new)
    lens = [300, 307, 290]
    cache, twin, slots, gen = build(bits, lens, 32, n_kv_heads, 128, torch.float16, 6, [(0, 3)], [280])
    run(cache, twin, slots, gen, n_heads, q_len, [min(q_len, 9)] * 3, [(0, 3)], [280])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("head_dim,dtype", [(64, torch.bfloat16), (96, torch.float16), (128, torch.bfloat16)])
def test_long(bits, head_dim, dtype):
    """One long sequence over all SMs, and a batch of unlike lengths."""
    cache, twin, slots, gen = build(bits, [70001], 64, 1, head_dim, dtype, 21)
    run(cache, twin, slots, gen, 5, 1)
    lens = [9000 - 811 * i for i in range(11)] + [3] * 20
    cache, twin, slots, gen = build(bits, lens, 16, 2, head_dim, dtype, 22)
    run(cache, twin, slots, gen, 8, 1)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("strength", [0.0, 1e-3, 12.0])
def test_logits(bits, strength):
    """Flat and sharp softmaxes, a scale of the caller's, layers."""
    lens = [900, 1025, 64]
    cache, twin, slots, gen = build(bits, lens, 64, 2, 128, torch.bfloat16, 31, n_layers=2)
    run(cache, twin, slots, gen, 6, 1, layer=1, strength=strength, scale=0.05 if strength else 0.0)


@pytest.mark.parametrize("bits", [4, 8])
def test_maximum_that_keeps_growing(bits):
    """Keys that get larger from tile to tile: the running maximum moves far, again and again; and the other way round."""
    for flip in (False, True):
        cache, twin, slots, gen = build(bits, [1500], 64, 1, 64, torch.bfloat16, 41)
        n = 1500
        size = torch.linspace(0.1, 40.0, n, device="cuda")
        x = torch.ones((1, 1, n, 64), device="cuda") * (size.flip(0) if flip else size)[:, None]
        K = x.to(torch.bfloat16)
        V = torch.randn((1, 1, n, 64), generator=gen, device="cuda").to(torch.bfloat16)
        cache.write(0, u32(slots), u32([n]), K, V)
        from quant_helpers import stored
        at = torch.arange(n, device="cuda")
        page, off = cache.table[slots[0]].long()[at // 64], at % 64
        twin.pool[0, page, :, off] = stored(K, bits)[0].transpose(0, 1)
        twin.pool[1, page, :, off] = stored(V, bits)[0].transpose(0, 1)
        Q = torch.full((1, 3, 1, 64), 0.5, dtype=torch.bfloat16, device="cuda")
        Q[0, 1] *= -1
        Q[0, 2] *= 0.01
        O = torch.empty_like(Q)
        cache.attend(0, Q, O, u32(slots))
        want, A = attention(twin, 0, Q, slots, [1])
        check_attention(O, want, A, n, 10.0)


@pytest.mark.parametrize("bits", [4, 8])
def test_wide_range_of_queries(bits):
    """Rows of very large and very small queries in one tile, values at the ends of what the cache holds."""
    cache, twin, slots, gen = build(bits, [333, 200], 16, 1, 64, torch.bfloat16, 51, spread=2.0 ** -6)
    Q = torch.randn((2, 4, 1, 64), generator=gen, device="cuda")
    Q *= torch.tensor([1.0, 2.0 ** -30, 2.0 ** 9, 2.0 ** -100], device="cuda")[None, :, None, None]
    Q = Q.to(torch.bfloat16)
    O = torch.empty_like(Q)
    cache.attend(0, Q, O, u32(slots))
    want, A = attention(twin, 0, Q, slots, [1, 1])
    check_attention(O, want, A, 333, 1.0)
    cache, twin, slots, gen = build(bits, [333, 200], 16, 1, 64, torch.bfloat16, 52, spread=8000.0)
    run(cache, twin, slots, gen, 4, 1, strength=1e-4)


@pytest.mark.parametrize("bits", [4, 8])
def test_rows_without_keys(bits):
    """A request that has more new tokens than tokens: its first rows see nothing."""
    cache, twin, slots, gen = build(bits, [3, 200, 0], 16, 2, 64, torch.bfloat16, 61)
    Q = torch.randn((3, 4, 8, 64), generator=gen, device="cuda").to(torch.bfloat16)
    O = torch.full_like(Q, float("nan"))
    cache.attend(0, Q, O, u32(slots), u32([8, 0, 2]))
    want, A = attention(twin, 0, Q, slots, [8, 0, 2])
    check_attention(O, want, A, 200, 6.0)
    assert not O[0, :, :5].any() and not O[1:].any()


@pytest.mark.parametrize("bits", [4, 8])
def test_faults(bits):
    """A page id out of range gives 0 for who reads it; bad slots, lengths and groups are left out and recorded."""
    lens = [300, 400, 500, 310, 320, 330]
    groups, shared = [(3, 6)], [300]
    cache, twin, slots, gen = build(bits, lens, 16, 2, 128, torch.bfloat16, 71, groups, shared)
    cache.table[slots[1], 20] = cache.n_pages
    cache.table[slots[2], 0] = -1
    Q = torch.randn((6, 4, 1, 128), generator=gen, device="cuda").to(torch.bfloat16)
    O = torch.full_like(Q, float("nan"))
    new = [1] * 6
    cache.attend(0, Q, O, u32(slots), u32(new), u32([3, 6]), u32([300]))
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    good = [s if i not in (1, 2) else -1 for i, s in enumerate(slots)]
    want, A = attention(twin, 0, Q, good, new)
    check_attention(O, want, A, 500, 6.0)
    assert not O[1:3].any()
    # An unsound id in the shared pages: the whole group.
    cache.table[slots[3], 2] = cache.n_pages + 5
    O.fill_(float("nan"))
    cache.attend(0, Q, O, u32(slots), u32(new), u32([3, 6]), u32([300]))
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    assert not O[3].any() and torch.isfinite(O).all()
    cache.table[slots[3], 2] = cache.table[slots[4], 2]
    # Groups that break their rules are passed over.
    for start in ([4, 2], [-1, 3], [0, 7]):
        O.fill_(float("nan"))
        cache.attend(0, Q, O, u32(good), u32(new), u32(start), u32([300]))
        assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
        check_attention(O, want, A, 500, 6.0)
    for bad_slot, bad_new in ((8, 1), (slots[0], 2), (slots[0], -1)):
        O.fill_(float("nan"))
        cache.attend(0, Q, O, u32([bad_slot] + good[1:]), u32([bad_new] + new[1:]))
        assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
        assert not O[0].any()
        check_attention(O[1:], want[1:], A[1:], 500, 6.0)


@pytest.mark.parametrize("bits", [4, 8])
def test_repeats_bit_for_bit_and_replays(bits):
    """The same call gives the same bits; a captured call follows new lengths; two streams with a cache object each."""
    lens = [5000, 3, 777, 12000]
    cache, twin, slots, gen = build(bits, lens, 64, 4, 128, torch.bfloat16, 81)
    Q = torch.randn((4, 16, 2, 128), generator=gen, device="cuda").to(torch.bfloat16)
    O, s, new = torch.empty_like(Q), u32(slots), u32([2, 1, 2, 1])
    cache.attend(0, Q, O, s, new)
    first = O.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attend(0, Q, O, s, new)
    for _ in range(20):
        O.fill_(0)
        g.replay()
        assert torch.equal(O, first)
    cache.lens.copy_(torch.clamp(cache.lens, max=900))
    new.copy_(u32([1, 1, 0, 2]))
    g.replay()
    want, A = attention(twin, 0, Q, slots, [1, 1, 0, 2])
    check_attention(O, want, A, 900, 6.0)
    other = serve.PagedCache.over(cache.pool, cache.table, cache.lens, cache.refs, bits, cache.page, cache.head_dim, cache.dtype)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(Q) for _ in range(2)]
    for st, c, o in zip(streams, (cache, other), outs):
        st.wait_stream(torch.cuda.current_stream())
        for _ in range(10):
            c.attend(0, Q, o, s, new, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], O) and torch.equal(outs[1], O)
    assert wise.wise_get_status() == wise.WISE_OK
