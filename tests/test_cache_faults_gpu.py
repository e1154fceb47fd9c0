"""Entries of the cache's lists that break the rules, and unused ones: they change nothing, and the sound entries of the
same call are done (integers and copied rows: every comparison is exact)."""
import random

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import u32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head_dim", [64, 96, 128])
@pytest.mark.parametrize("batch,q_len,n_kv_heads", [(2, 1, 1), (5, 3, 1), (33, 1, 1), (40, 1, 3), (300, 2, 2),
                                                    (700, 1, 1)])
def test_a_slot_that_a_write_lists_twice_is_not_written(head_dim, batch, q_len, n_kv_heads):
    """Whichever blocks the two entries fall to; entries without a slot may be as many as they like."""
    r = random.Random(batch + head_dim)
    page, n_slots = 16, batch + 3
    cache = serve.PagedCache(1, n_slots, n_kv_heads, page, head_dim, n_slots, 1)
    cache.table.copy_(torch.arange(n_slots, dtype=torch.int32, device="cuda")[:, None])
    cache.lens.fill_(page)
    cache.refs.fill_(1)
    K, V = (torch.randn((batch, n_kv_heads, q_len, head_dim), device="cuda").bfloat16() for _ in range(2))
    slots = r.sample(range(n_slots), batch)
    lists = [slots, [slots[1]] + slots[1:], slots[:-1] + [slots[0]]]
    if batch > 5:
        some = list(slots)
        for a, b in ((3, batch - 2), (batch // 2, batch // 2 + 1), (0, 1), (1, 5)):
            some[a] = some[b]
        for a in (2, batch - 1):
            some[a] = -1
        lists += [some, [slots[0]] * batch, [-1] * batch]
    for at in lists:
        n_new = [r.randint(0, q_len) for _ in at]
        want = cache.pool.normal_().clone()
        faults = False
        for b, s in enumerate(at):
            if s >= 0 and at.count(s) > 1:
                faults = True
            elif s >= 0 and n_new[b]:
                for plane, x in ((0, K), (1, V)):
                    want[plane, s, :, page - n_new[b]:] = x[b, :, :n_new[b]]
        cache.write(0, u32(at), u32(n_new), K, V)
        assert wise.wise_get_status() == (wise.WISE_ERR_BAD_CACHE if faults else wise.WISE_OK)
        assert torch.equal(cache.pool.view(torch.int16), want.view(torch.int16))


def cache_of(rows, lens, n_pages=24, page=16, max_pages=4, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16):
    """A cache whose slot s holds lens[s] tokens in pages rows[s]."""
    cache = serve.PagedCache(1, n_pages, n_kv_heads, page, head_dim, len(rows), max_pages, dtype)
    cache.pool.copy_(torch.randn(cache.pool.shape, device="cuda"))
    refs = [0] * n_pages
    for s, row in enumerate(rows):
        cache.table[s, :len(row)] = u32(row)
        for g in row:
            if 0 <= g < n_pages:
                refs[g] += 1
    cache.lens.copy_(u32(lens))
    cache.refs.copy_(u32(refs))
    return cache


def state(cache):
    return cache.table.tolist(), cache.lens.tolist(), cache.refs.tolist()


FAULTY_IDS = [-1, 24, 2 ** 31 - 1, -2 ** 31]


@pytest.mark.parametrize("bad", FAULTY_IDS)
@pytest.mark.parametrize("at", [0, 1, 2])
def test_a_fork_from_or_over_a_faulty_page_id_changes_nothing(bad, at):
    row = [3, 4, 5]
    row[at] = bad
    # Slot 0 is faulty, slots 1 and 2 are sound, 3 and 4 hold something, 5 is empty.
    rows = [row, [6, 7], [8], [9, 10], [11], []]
    lens = [40, 20, 3, 32, 16, 0]
    cache = cache_of(rows, lens)
    before = state(cache)
    cache.fork(u32([0]), u32([3]))                       # from the faulty row
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    assert state(cache) == before
    cache.fork(u32([1]), u32([0]))                       # over the faulty row
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    assert state(cache) == before
    cache.fork(u32([0, 1]), u32([4, 5]))                 # beside a sound entry
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    table, lens2, refs = state(cache)
    assert lens2 == [40, 20, 3, 32, 16, 20] and table[5][:2] == [6, 7] and table[:5] == before[0][:5]
    assert refs == [before[2][g] + (g in (6, 7)) for g in range(24)]


def test_a_fork_does_not_look_past_the_lengths():
    """Entries behind a sequence's pages mean nothing, whatever they hold."""
    cache = cache_of([[3], [4], []], [16, 9, 0])
    cache.table[0, 1:] = -7
    cache.table[1, 1:] = 1 << 30
    cache.fork(u32([0]), u32([1]))
    assert wise.wise_get_status() == wise.WISE_OK
    assert cache.lens.tolist() == [16, 16, 0] and cache.table[1, 0].item() == 3 and cache.refs[3].item() == 2


@pytest.mark.parametrize("bad", FAULTY_IDS)
@pytest.mark.parametrize("at,drop", [(0, 40), (1, 25), (2, 10), (0, 1 << 30), (2, 40)])
def test_a_drop_over_a_faulty_page_id_changes_nothing(bad, at, drop):
    row = [3, 4, 5]
    row[at] = bad
    cache = cache_of([row, [6, 7]], [40, 20])
    before = state(cache)
    cache.drop(u32([0, 1]), u32([drop, 10]))
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    table, lens, refs = state(cache)
    assert table == before[0] and lens == [40, 10]
    assert refs == [before[2][g] - (g == 7) for g in range(24)]


def test_a_drop_does_not_look_past_what_it_releases():
    """Pages that stay are not the call's concern, nor are entries behind the length."""
    cache = cache_of([[-1, 4, 5]], [40])
    cache.table[0, 3] = 1 << 30
    cache.drop(u32([0]), u32([10]))
    assert wise.wise_get_status() == wise.WISE_OK
    assert cache.lens.tolist() == [30] and cache.refs[5].item() == 0 and cache.refs[4].item() == 1


@pytest.mark.parametrize("src,dst", [([0, -1], [2, 2]), ([-5, 0], [2, 2]), ([0, 2], [2, -1]), ([0, -1, 1], [2, 0, 3]),
                                     ([-1, -1, 0], [2, 2, 2]), ([0, 2, 1], [2, -3, 3])])
def test_unused_entries_of_a_fork_are_passed_over(src, dst):
    """What stands beside a negative slot is not looked at: it neither lists a slot twice nor makes one a source."""
    rows, lens = [[3, 4], [5], [6], []], [20, 7, 2, 0]
    cache = cache_of(rows, lens)
    for s, d in zip(src, dst):
        if s >= 0 and d >= 0:
            rows[d], lens[d] = rows[s], lens[s]
    refs = [sum(row.count(g) for row in rows) for g in range(24)]
    cache.fork(u32(src), u32(dst))
    assert wise.wise_get_status() == wise.WISE_OK
    table, got, got_refs = state(cache)
    assert got == lens and got_refs == refs
    assert [t[:len(r)] for t, r in zip(table, rows)] == rows


def test_lengths_next_to_the_largest_integer():
    """Nothing is read, written or changed for a sequence whose length cannot be."""
    K = torch.randn((1, 2, 2, 64), device="cuda").bfloat16()
    for length in ((1 << 31) - 1, -(1 << 31), (1 << 31) - 65, 65):
        cache = cache_of([[3, 4, 5], []], [length, 0])
        pool, before = cache.pool.clone(), state(cache)
        for call in (lambda: cache.fork(u32([0]), u32([1])), lambda: cache.fork(u32([1]), u32([0])),
                     lambda: cache.extend(u32([0]), u32([30])), lambda: cache.write(0, u32([0]), None, K, K),
                     lambda: cache.drop(u32([0]), u32([1 << 30]))):
            call()
            assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
            assert state(cache) == before and torch.equal(cache.pool.view(torch.int16), pool.view(torch.int16))
