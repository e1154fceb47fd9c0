"""Calls on caches in 8 or 4 bits (reading: of 16 too) that take the less usual ways: memory aligned to 16 bytes only, batches
large enough for a warp to take whole rows, pages past 2^32 bytes, queries and table entries that nobody reads."""
import random

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from quant_helpers import build, check_attention, stored
from serve_helpers import attention, u32
from test_quant_attn_gpu import run

pytestmark = pytest.mark.gpu


def at_16(shape, dtype, fill=None):
    """A contiguous tensor whose memory begins 16 bytes behind an aligned one, and the elements around it."""
    n, edge = 1, 16 // dtype.itemsize
    for x in shape:
        n *= x
    room = torch.full((n + 2 * edge,), 7.0, dtype=dtype, device="cuda")
    t = room[edge:edge + n].view(shape)
    assert t.data_ptr() % 32 == 16 and t.is_contiguous()
    if fill is not None:
        t.copy_(fill)
    return t, (room[:edge], room[edge + n:])


def sequences(bits, page, kv, dim, dtype, batch, most, seed):
    """A cache of `batch` sequences that have grown by rows of their own each, and what it then stands for: a call has
    written `before` tokens, the next one `new` more; K and V of these calls."""
    r = random.Random(seed)
    before = [r.choice([0, 1, 15, 16, 31, 33, r.randint(0, 70)]) for _ in range(batch)]
    new = [r.choice([0, 1, most, r.randint(1, most)]) for _ in range(batch)]
    max_pages = -(-(max(before) + most) // page)
    c = serve.PagedCache(1, sum(-(-(a + b) // page) for a, b in zip(before, new)) + 1, kv, page, dim, batch, max_pages, dtype,
                         bits=bits)
    if bits == 16:
        c.pool.fill_(float("nan"))
    else:
        c.pool.random_(0, 256)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    parts = [torch.randn((2, batch, kv, n, dim), generator=gen, device="cuda").to(dtype) for n in (max(max(before), 1), most)]
    order = r.sample(range(batch), batch)
    return c, order, before, new, parts


def what_it_holds(bits, before, new, parts):
    return [torch.cat([stored(p[:, i, :, :n[i]], bits) if bits < 16 else p[:, i, :, :n[i]].double()
                       for p, n in zip(parts, (before, new))], 2) for i in range(len(new))]


@pytest.mark.parametrize("bits", [4, 8, 16])
@pytest.mark.parametrize("batch,most,page,dim,dtype", [(3, 40, 16, 96, torch.float16), (2, 5, 64, 128, torch.bfloat16),
                                                       (64, 150, 32, 64, torch.bfloat16), (64, 150, 16, 96, torch.float16)])
def test_memory_aligned_to_16_bytes(bits, batch, most, page, dim, dtype):
    """K and V that begin 16 bytes behind a multiple of 32, stored and read; nothing beside them is written."""
    kv = 8
    c, order, before, new, parts = sequences(bits, page, kv, dim, dtype, batch, most, seed=batch + page)
    s = u32(order)
    for x, n in zip(parts, (before, new)):
        granted = c.extend(s, u32(n))
        K, V = (at_16(x.shape[1:], dtype, y)[0] for y in x)
        c.write(0, s, granted, K, V)
    rows = max(a + b for a, b in zip(before, new))
    (K, ends), (V, more) = (at_16((batch, kv, rows, dim), dtype, float("nan") * torch.ones(1, device="cuda")) for _ in range(2))
    c.read(0, K, V, s)
    for i, want in enumerate(what_it_holds(bits, before, new, parts)):
        n = want.shape[2]
        assert torch.equal(torch.stack([K[i, :, :n], V[i, :, :n]]).double(), want)
        assert not K[i, :, n:].any() and not V[i, :, n:].any()
    assert all(bool((x == 7).all()) for x in ends + more)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_heads", [8, 40])
def test_queries_aligned_to_16_bytes(bits, n_heads):
    cache, twin, slots, gen = build(bits, [300, 77, 1000], 32, 2, 96, torch.bfloat16, 13)
    Q, first = run(cache, twin, slots, gen, n_heads, 1)
    q, _ = at_16(Q.shape, Q.dtype, Q)
    O, ends = at_16(Q.shape, Q.dtype)
    cache.attend(0, q, O, u32(slots))
    assert torch.equal(O, first) and all(bool((x == 7).all()) for x in ends)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8, 16])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim,dtype", [(64, torch.bfloat16), (96, torch.float16), (128, torch.bfloat16)])
def test_batches_in_which_a_warp_takes_whole_rows(bits, page, dim, dtype):
    """More spans of 32 tokens than 16 for each SM: ragged sequences behind others, stored, and read in ragged spans."""
    kv, batch, most = 8, 48, 300
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert batch * kv * (most // 32) >= 16 * sms
    c, order, before, new, parts = sequences(bits, page, kv, dim, dtype, batch, most, seed=page + dim)
    s = u32(order)
    for x, n in zip(parts, (before, new)):
        c.write(0, s, c.extend(s, u32(n)), x[0].contiguous(), x[1].contiguous())
    r = random.Random(page)
    first = [r.choice([0, r.randint(0, a + b)]) for a, b in zip(before, new)]
    count = [r.choice([0, most, r.randint(0, most)]) for _ in first]
    K = torch.full((batch, kv, most, dim), float("nan"), dtype=dtype, device="cuda")
    V = K.clone()
    c.read(0, K, V, s, u32(first), u32(count))
    for i, all_of_it in enumerate(what_it_holds(bits, before, new, parts)):
        want = all_of_it[:, :, first[i]:first[i] + count[i]]
        n = want.shape[2]
        assert torch.equal(torch.stack([K[i, :, :n], V[i, :, :n]]).double(), want), i
        assert not K[i, :, n:].any() and not V[i, :, n:].any()
    assert wise.wise_get_status() == wise.WISE_OK


class Shifted:
    """The last pages of a cache, for serve_helpers.attention: values [2, pages, kv, page, dim] of pages `first` .."""

    def __init__(self, cache, pool, first):
        self.pool, self.table, self.lens = pool, cache.table - first, cache.lens
        self.page, self.n_kv_heads = cache.page, cache.n_kv_heads


@pytest.mark.parametrize("bits,n_pages", [(4, 30000), (8, 16000)])
def test_pages_past_32_bits_of_bytes(bits, n_pages):
    """Storing, reading and attention (of few and of many rows, with and without a shared prefix) at the end of a pool of
    more than 2^32 bytes."""
    page, dim, kv, batch, n = 128, 128, 8, 40, 300
    used = 3 * batch
    c = serve.PagedCache(1, n_pages, kv, page, dim, batch, 3, torch.bfloat16, bits=bits)
    assert (n_pages - used) * c.pool.stride(1) > 2 ** 32
    c.table.copy_((n_pages - 1 - torch.arange(used, device="cuda")).int().view(batch, 3))
    c.table[:, 0] = c.table[0, 0]  # the first page is shared
    c.refs[-used:] = 1
    gen = torch.Generator(device="cuda").manual_seed(bits)
    x = torch.randn((2, batch, kv, n, dim), generator=gen, device="cuda").bfloat16()
    x[:, :, :, :page] = x[:, :1, :, :page]
    slots = list(range(batch))
    c.lens.fill_(n)
    one = u32([n] + [n - page] * (batch - 1))  # the others write behind the shared page
    own = torch.zeros_like(x)
    own[:, 0] = x[:, 0]
    own[:, 1:, :, :n - page] = x[:, 1:, :, page:]
    c.write(0, u32(slots), one, own[0].contiguous(), own[1].contiguous())
    c.refs[c.table[0, 0].long()] = batch
    got = torch.empty_like(x)
    c.read(0, got[0], got[1], u32(slots))
    want = stored(x, bits)
    assert torch.equal(got.double(), want)
    pool = torch.zeros((2, used, kv, page, dim), dtype=torch.float64, device="cuda")
    twin = Shifted(c, pool, n_pages - used)
    for p in range(3):
        m = min(page, n - p * page)
        pool[:, twin.table[:, p].long(), :, :m] = want[:, :, :, p * page:p * page + m]
    for heads in (8, 160):
        Q = torch.randn((batch, heads, 1, dim), generator=gen, device="cuda").bfloat16()
        ref, A = attention(twin, 0, Q, slots, [1] * batch)
        for groups in ((None, None), (u32([0, batch]), u32([200]))):
            O = torch.full_like(Q, float("nan"))
            c.attend(0, Q, O, u32(slots), None, *groups)
            check_attention(O, ref, A, n, float(pool.abs().max()))
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_heads,q_len", [(8, 1), (8, 4), (20, 2), (40, 3), (80, 1)])
def test_faults_in_a_shared_prefix(bits, n_heads, q_len):
    """A page id out of range there gives 0 for all requests of the group and leaves the others alone, whether the group's
    part is joined with own parts or not; the table rows that nobody reads the prefix through may hold anything."""
    lens = [300, 400, 500, 310, 288, 1700, 640, 333]
    groups, shared = [(3, 6), (6, 8)], [290, 320]
    cache, twin, slots, gen = build(bits, lens, 16, 2, 128, torch.bfloat16, 7 * q_len, groups, shared)
    new = [min(1 + i % q_len, n) for i, n in enumerate(lens)]
    Q = torch.randn((8, n_heads, q_len, 128), generator=gen, device="cuda").bfloat16()
    want, A = attention(twin, 0, Q, slots, new)
    start, spans = u32([3, 6, 8]), u32(shared)

    def check(faulty, status):
        O = torch.full_like(Q, float("nan"))
        cache.attend(0, Q, O, u32(slots), u32(new), start, spans)
        assert wise.wise_get_status() == status
        good = [i for i in range(8) if i not in faulty]
        check_attention(O[good], want[good], A[good], 1700, float(twin.pool.abs().max()))
        assert not O[faulty].any()

    check([], wise.WISE_OK)
    lead = n_heads // 2 * q_len <= 32  # rows above 32 a kv head: everybody reads the prefix by itself
    sound = cache.table.clone()
    cache.table[slots[3], 2] = cache.n_pages + 5
    check([3, 4, 5] if lead else [3], wise.WISE_ERR_BAD_CACHE)
    cache.table.copy_(sound)
    cache.table[slots[4], 2] = cache.table[slots[7], 0] = -9
    check([] if lead else [4, 7], wise.WISE_OK if lead else wise.WISE_ERR_BAD_CACHE)
    cache.table.copy_(sound)
    cache.table[slots[5], 1600 // 16] = cache.n_pages  # a page of its own
    check([5], wise.WISE_ERR_BAD_CACHE)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,n_heads,q_len", [(64, 4, 4), (96, 4, 5), (128, 16, 4), (96, 30, 4)])
def test_queries_that_nobody_asked_may_hold_anything(bits, dtype, dim, n_heads, q_len):
    """Rows past n_new, of unused entries and of empty sequences hold NaN, infinities and the type's extremes: they give 0,
    and the other rows the same bits as beside zeros."""
    lens = [200, 333, 0, 270, 260, 300, 259]
    groups, shared = [(3, 7)], [250]
    cache, twin, slots, gen = build(bits, lens, 32, 2, dim, dtype, dim + q_len, groups, shared)
    new = [1, 0, 2, q_len, 2, 1, q_len]
    slots[5] = -1
    Q = torch.randn((7, n_heads, q_len, dim), generator=gen, device="cuda").to(dtype)
    asked = torch.zeros((7, 1, q_len, 1), dtype=torch.bool, device="cuda")
    for i, n in enumerate(new):
        asked[i, :, :n if lens[i] and slots[i] >= 0 else 0] = True
    top = float(torch.finfo(dtype).max)
    junk = torch.tensor([float("nan"), float("inf"), -float("inf"), top, -top, 1e-5], device="cuda")
    junk = junk[torch.randint(0, 6, Q.shape, generator=gen, device="cuda")].to(dtype)
    want, A = attention(twin, 0, torch.where(asked, Q, 0), slots, new)
    for start, spans in ((None, None), (u32([3, 7]), u32([250]))):
        outs = []
        for other in (torch.zeros_like(Q), junk):
            O = torch.full_like(Q, float("nan"))
            cache.attend(0, torch.where(asked, Q, other), O, u32(slots), u32(new), start, spans)
            outs.append(O)
        assert torch.equal(outs[0], outs[1]) and not outs[1][~asked.expand_as(Q)].any()
        check_attention(outs[1], want, A, 333, float(twin.pool.abs().max()))
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_nan_leaves_the_others_of_its_group_alone(bits, dtype):
    """NaN of either sign in keys and values: every finite value, of the same 16 too, is stored as it would be without it."""
    c = serve.PagedCache(1, 6, 3, 32, 96, 2, 3, dtype, bits=bits)
    gen = torch.Generator(device="cuda").manual_seed(bits)
    x = torch.randn((2, 2, 3, 45, 96), generator=gen, device="cuda").to(dtype)
    is_nan = torch.rand(x.shape, generator=gen, device="cuda") < 0.1
    is_nan[..., 3, :16] = True  # a group of nothing else
    bad = torch.full_like(x, float("nan"))
    K, V = torch.where(is_nan, torch.where(torch.rand(x.shape, generator=gen, device="cuda") < 0.5, bad, -bad), x)
    s = u32([1, 0])
    c.write(0, s, c.extend(s, u32([45, 45])), K.contiguous(), V.contiguous())
    got = torch.empty_like(x)
    c.read(0, got[0], got[1], s)
    want = stored(torch.where(is_nan, 0, x), bits)
    assert torch.equal(torch.where(is_nan, 0, got.double()), want)
    assert wise.wise_get_status() == wise.WISE_OK
