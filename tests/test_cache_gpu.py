"""The paged cache's operations against lists (integers and copied rows: every
comparison is exact)."""
import random

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import ListCache, u32

pytestmark = pytest.mark.gpu


def make(n_layers=2, n_pages=40, n_kv_heads=3, page=16, head_dim=64, n_slots=12, max_pages=6, dtype=torch.bfloat16):
    cache = serve.PagedCache(n_layers, n_pages, n_kv_heads, page, head_dim, n_slots, max_pages, dtype)
    cache.pool.copy_(torch.randn(cache.pool.shape, device="cuda"))
    return cache, ListCache(n_pages, page, n_slots, max_pages)


def tokens_of(cache, s):
    """What the sequence in slot s holds: [n_layers * 2, n_kv_heads, len, head_dim]."""
    n = int(cache.lens[s])
    at = torch.arange(n, device="cuda")
    return cache.pool[:, cache.table[s].long()[at // cache.page], :, at % cache.page].permute(1, 2, 0, 3)


def grow(cache, model, contents, slots, n_new):
    """extend + write on both sides; contents[s] follows the tokens of every sequence."""
    want, _ = model.extend(slots, n_new)
    granted = cache.extend(u32(slots), u32(n_new))
    assert granted.tolist() == want
    q_len = max(n_new + [1])
    shape = (len(slots), cache.n_kv_heads, q_len, cache.head_dim)
    new = [torch.randn(shape, device="cuda").to(cache.dtype) for _ in range(2 * cache.n_layers)]
    for layer in range(cache.n_layers):
        cache.write(layer, u32(slots), granted, new[2 * layer], new[2 * layer + 1])
    for b, s in enumerate(slots):
        if s >= 0 and want[b]:
            contents[s] = torch.cat([contents[s], torch.stack([x[b, :, :want[b]] for x in new])], 2)
    model.matches(cache)


def empty_contents(cache):
    return [torch.empty((2 * cache.n_layers, cache.n_kv_heads, 0, cache.head_dim), dtype=cache.dtype, device="cuda")
            for _ in range(cache.n_slots)]


def same_contents(cache, contents):
    for s in range(cache.n_slots):
        got = tokens_of(cache, s)
        assert torch.equal(got.view(torch.int16), contents[s].view(torch.int16)), s


@pytest.mark.parametrize("page,head_dim,dtype,n_kv_heads", [
    (16, 64, torch.bfloat16, 3), (32, 96, torch.float16, 1), (64, 128, torch.bfloat16, 2), (128, 96, torch.bfloat16, 5)])
def test_random_histories(page, head_dim, dtype, n_kv_heads):
    """Many steps of growing, forking, dropping and compacting: bookkeeping equal to the lists, and every
    sequence still holds exactly the tokens that were written to it."""
    r = random.Random(page)
    cache, model = make(page=page, head_dim=head_dim, dtype=dtype, n_kv_heads=n_kv_heads)
    contents = empty_contents(cache)
    for step in range(30):
        what = r.choice(["grow", "grow", "fork", "drop", "compact"])
        slots = r.sample(range(cache.n_slots), r.randint(1, 8))
        if what == "grow":
            grow(cache, model, contents, slots, [r.choice([0, 1, 1, 3, page, page + 1]) for _ in slots])
        elif what == "fork":
            src = [r.choice(range(cache.n_slots)) for _ in slots]
            slots = [s for s in slots if s not in src]
            src = src[:len(slots)]
            model.fork(src, slots)
            cache.fork(u32(src), u32(slots))
            for a, b in zip(src, slots):
                contents[b] = contents[a]
        elif what == "drop":
            n = [r.choice([0, 1, 2, page, 1 << 30]) for _ in slots]
            model.drop(slots, n)
            cache.drop(u32(slots), u32(n))
            for s, k in zip(slots, n):
                contents[s] = contents[s][:, :, :max(0, contents[s].shape[2] - k)]
        else:
            remap, n_live, _ = model.compact()
            got_map, got_live = cache.compact()
            assert got_map.tolist() == remap and got_live.tolist() == [n_live]
        model.matches(cache)
        same_contents(cache, contents)
    status = wise.wise_get_status()
    assert status == (wise.WISE_ERR_NO_PAGES if model.starved else wise.WISE_OK)


def test_shared_tail_is_copied_and_only_its_rows():
    cache, model = make(page=32)
    contents = empty_contents(cache)
    grow(cache, model, contents, [0], [32 + 7])
    before = cache.pool.clone()
    model.fork([0, 0], [3, 4])
    cache.fork(u32([0, 0]), u32([3, 4]))
    _, copies = model.extend([0, 3, 4], [1, 2, 0])
    cache.extend(u32([0, 3, 4]), u32([1, 2, 0]))
    model.matches(cache)
    for a, b, rows in copies:
        before[:, b, :, :rows] = before[:, a, :, :rows]
    assert len(copies) == 2 and torch.equal(cache.pool.view(torch.int16), before.view(torch.int16))


def test_a_full_shared_page_is_not_copied():
    cache, model = make()
    grow(cache, model, empty_contents(cache), [0], [32])
    model.fork([0], [1])
    cache.fork(u32([0]), u32([1]))
    _, copies = model.extend([0, 1], [1, 1])
    cache.extend(u32([0, 1]), u32([1, 1]))
    assert copies == []
    model.matches(cache)
    assert cache.refs[cache.table[0, 0].item()].item() == 2


def test_pages_run_out_entry_by_entry():
    cache, model = make(n_pages=5, n_slots=6, max_pages=4)
    grow(cache, model, empty_contents(cache), [0, 1], [16, 10])   # 3 pages left
    want, _ = model.extend([2, 3, 1, 0, 4], [33, 1, 6, 1, 0])     # 3 pages; none for 3; 1 fits its page; none for 0
    got = cache.extend(u32([2, 3, 1, 0, 4]), u32([33, 1, 6, 1, 0]))
    assert got.tolist() == want == [33, 0, 6, 0, 0]
    model.matches(cache)
    assert wise.wise_get_status() == wise.WISE_ERR_NO_PAGES
    want, _ = model.extend([1], [49])   # more than max_pages
    assert cache.extend(u32([1]), u32([49])).tolist() == want == [0]
    assert wise.wise_get_status() == wise.WISE_ERR_NO_PAGES
    model.matches(cache)


def test_faulty_entries_change_nothing():
    cache, model = make(n_slots=5)
    contents = empty_contents(cache)
    grow(cache, model, contents, [0, 1], [20, 5])
    for name, a, b in (("fork", [0, 0, 1], [2, 2, 3]), ("fork", [0, 2], [2, 4]), ("fork", [0], [0]),
                       ("fork", [0, 9, -1, 0], [9, 1, 2, -3]), ("drop", [0, 0, 7, -1], [1, 2, 3, 4]),
                       ("drop", [1], [-1]), ("extend", [1, 1, 5, -2, 0], [1, 1, 1, 1, 1]), ("extend", [0], [-4])):
        faults = model.faults
        getattr(model, name)(a, b)
        getattr(cache, name)(u32(a), u32(b))
        model.matches(cache)
        assert model.faults > faults and wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE, (name, a, b)


def test_faulty_tables_and_lengths_stay_in_bounds():
    """Page ids, lengths and counts that no call leaves behind: nothing is read or written out of range, and the
    status says so."""
    cache, _ = make(n_slots=4, max_pages=3, n_pages=8)
    guard = cache.pool.clone()
    K = torch.randn((1, cache.n_kv_heads, 2, cache.head_dim), device="cuda").bfloat16()
    for lens, row in ((20, [-1, -7, 0]), (20, [8, 1 << 30, 0]), (49, [0, 1, 2]), (-3, [0, 1, 2]), (1 << 31 - 1, [0, 1, 2])):
        calls = (lambda: cache.fork(u32([0]), u32([1])), lambda: cache.extend(u32([0]), u32([30])),
                 lambda: cache.write(0, u32([0]), None, K, K), lambda: cache.drop(u32([0]), u32([1 << 30])),
                 lambda: cache.compact())
        for call in calls:
            cache.table.zero_()
            cache.refs.zero_()
            cache.lens.zero_()
            cache.table[0] = u32(row)
            cache.lens[0] = lens
            call()
            assert wise.wise_get_status() in (wise.WISE_ERR_BAD_CACHE, wise.WISE_ERR_NO_PAGES), (lens, row)
            assert torch.equal(cache.pool.view(torch.int16), guard.view(torch.int16))


def test_write_leaves_shared_pages_alone():
    cache, model = make()
    grow(cache, model, empty_contents(cache), [0], [20])
    cache.fork(u32([0]), u32([1]))
    before = cache.pool.clone()
    K = torch.randn((1, cache.n_kv_heads, 1, cache.head_dim), device="cuda").bfloat16()
    cache.write(0, u32([1]), u32([1]), K, K)
    assert torch.equal(cache.pool.view(torch.int16), before.view(torch.int16))
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE


@pytest.mark.parametrize("n_pages", [1, 31, 1024, 1025, 5000, 70001])
@pytest.mark.parametrize("density", [0.0, 0.02, 0.5, 1.0])
def test_compact_over_many_pages(n_pages, density):
    """Prefix sums over pools below, at and above one block's width; tables of one page each."""
    r = random.Random(n_pages)
    n_slots = min(n_pages, 3000)
    cache = serve.PagedCache(1, n_pages, 1, 16, 64, n_slots, 1)
    cache.pool.copy_(torch.randn(cache.pool.shape, device="cuda"))
    model = ListCache(n_pages, 16, n_slots, 1)
    live = sorted(r.sample(range(n_pages), int(round(density * n_slots))))
    r.shuffle(live)
    for s, g in enumerate(live):
        model.rows[s], model.lens[s], model.refs[g] = [g], 1 + s % 16, 1
    cache.table.copy_(u32([[row[0] if row else 0] for row in model.rows]))
    cache.lens.copy_(u32(model.lens))
    cache.refs.copy_(u32(model.refs))
    before = cache.pool.clone()
    remap, n_live, moves = model.compact()
    got_map, got_live = cache.compact()
    assert got_live.item() == n_live and got_map.tolist() == remap
    model.matches(cache)
    for a, b in moves:
        before[:, b] = before[:, a]
    assert torch.equal(cache.pool.view(torch.int16), before.view(torch.int16))
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("n,n_pages", [(1, 1), (33, 1000), (1500, 3000), (2500, 6000)])
def test_extend_over_many_entries(n, n_pages):
    """Lists and pools longer than one block: the lowest free pages in list order."""
    r = random.Random(n)
    cache = serve.PagedCache(1, n_pages, 1, 16, 64, n, 4)
    model = ListCache(n_pages, 16, n, 4)
    taken = r.sample(range(n_pages), n_pages // 3)
    for g in taken:
        model.refs[g] = 1
    cache.refs.copy_(u32(model.refs))
    slots = r.sample(range(n), n)
    add = [r.randint(0, 40) for _ in slots]
    want, _ = model.extend(slots, add)
    assert cache.extend(u32(slots), u32(add)).tolist() == want
    model.matches(cache)
    wise.wise_get_status()


def test_offsets_past_32_bits():
    """A pool whose planes exceed 2^32 bytes: rows on its last pages are written, copied and moved."""
    n_pages = (1 << 32) // (8 * 128 * 128 * 2) + 100
    cache = serve.PagedCache(1, n_pages, 8, 128, 128, 4, 4)
    model = ListCache(n_pages, 128, 4, 4)
    model.refs[:n_pages - 6] = [1] * (n_pages - 6)
    cache.refs.copy_(u32(model.refs))
    contents = empty_contents(cache)
    grow(cache, model, contents, [0], [130])
    model.fork([0], [1])
    cache.fork(u32([0]), u32([1]))
    contents[1] = contents[0]
    grow(cache, model, contents, [1], [3])
    same_contents(cache, contents)
    for g in range(50):
        model.refs[g] = 0
    cache.refs.copy_(u32(model.refs))
    remap, n_live, _ = model.compact()
    got, live = cache.compact()
    assert live.item() == n_live and got.tolist() == remap
    model.matches(cache)
    same_contents(cache, contents)


def test_refusals_of_the_binding():
    cache, _ = make()
    ok = u32([0])
    with pytest.raises(ValueError):
        cache.fork(ok, u32([1, 2]))
    with pytest.raises(ValueError):
        cache.extend(ok.long(), ok)
    with pytest.raises(ValueError):
        cache.drop(ok, ok.cpu())
    with pytest.raises(ValueError):
        cache.write(0, ok, None, torch.zeros((1, 3, 1, 64), device="cuda"), torch.zeros((1, 3, 1, 64), device="cuda"))
    with pytest.raises(ValueError):
        wise.wise_kv_compact(cache, u32([0] * cache.n_pages), ok, torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(wise.WiseError):
        serve.PagedCache(1, 4, 1, 24, 64, 2, 2).drop(ok, ok)
    with pytest.raises(ValueError):
        serve.PagedCache.over(cache.pool[:, ::2], cache.table, cache.lens, cache.refs)


def test_on_another_stream():
    """Calls on a side stream while the default stream is busy: buffers made by the calls belong to that stream."""
    cache, model = make(n_pages=3000, n_slots=64, max_pages=40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    slots = u32(list(range(64)))
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for k in range(6):
        n_new = [(s * 7 + k) % 50 for s in range(64)]
        with torch.cuda.stream(side):
            add = u32(n_new)
        want, _ = model.extend(list(range(64)), n_new)
        got.append((cache.extend(slots, add, stream=side), want))
        torch.randn(1 << 20, device="cuda")
    remap, n_live, _ = model.compact()
    out = cache.compact(stream=side)
    side.synchronize()
    for g, w in got:
        assert g.tolist() == w
    assert out[0].tolist() == remap and out[1].item() == n_live
    model.matches(cache)
