"""Attention over the paged cache against its definition in fp64."""
import random

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import attention, check_attention, u32

pytestmark = pytest.mark.gpu


def build(lens, shared, groups, page, n_kv_heads, head_dim, dtype, seed, spare_slots=2, poison=True, n_layers=1):
    """A cache whose requests have the given lengths; the requests of group g (start, end) share the pages of
    their first shared[g] tokens.  Rows that hold no token are NaN."""
    r = random.Random(seed)
    B = len(lens)
    slots = r.sample(range(B + spare_slots), B)
    max_pages = max([-(-n // page) for n in lens] + [1]) + 1
    rows, need = {}, 0
    for g, (a, b) in enumerate(groups):
        for i in range(a, b):
            rows[i] = -(-lens[i] // page)
    n_pages = sum(-(-n // page) for n in lens) + 3
    ids = r.sample(range(n_pages), n_pages)
    table = torch.randint(0, n_pages, (B + spare_slots, max_pages)).tolist()   # unused entries mean nothing
    length, refs = [0] * (B + spare_slots), [0] * n_pages
    common = {}
    for g, (a, b) in enumerate(groups):
        whole = min([lens[i] for i in range(a, b)] + [shared[g]]) // page
        pages = [ids.pop() for _ in range(whole)]
        for i in range(a, b):
            common[i] = pages
    for i, n in enumerate(lens):
        row = list(common.get(i, []))[:-(-n // page)]
        row += [ids.pop() for _ in range(-(-n // page) - len(row))]
        table[slots[i]][:len(row)] = row
        length[slots[i]] = n
        for g in row:
            refs[g] += 1
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pool = torch.randn((2 * n_layers, n_pages, n_kv_heads, page, head_dim), generator=gen, device="cuda").to(dtype)
    cache = serve.PagedCache.over(pool, u32(table), u32(length), u32(refs))
    if poison:
        used = torch.zeros((n_pages, page), dtype=torch.bool, device="cuda")
        for s, n in enumerate(length):
            at = torch.arange(n, device="cuda")
            used[cache.table[s].long()[at // page], at % page] = True
        bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda").to(dtype)
        fill = bad[torch.randint(0, 3, (n_pages, 1, page, head_dim), generator=gen, device="cuda")]
        pool.copy_(torch.where(used[None, :, None, :, None], pool, fill[None]))
    return cache, slots, gen


def run(cache, slots, gen, n_heads, q_len, n_new=None, groups=None, shared=None, scale=0.0, layer=0, strength=1.5):
    B = len(slots)
    Q = (torch.randn((B, n_heads, q_len, cache.head_dim), generator=gen, device="cuda") * strength).to(cache.dtype)
    O = torch.full_like(Q, float("nan"))
    start = None if groups is None else u32([groups[0][0]] + [b for _, b in groups])
    cache.attend(layer, Q, O, u32(slots), None if n_new is None else u32(n_new), start,
                 None if shared is None else u32(shared), scale)
    new = n_new if n_new is not None else [q_len] * B
    want, A = attention(cache, layer, Q, slots, new, scale)
    n_keys = max([cache.lens.tolist()[s] for s in slots if s >= 0] + [0])
    check_attention(O, want, A, n_keys, 6.0)
    return Q, O


@pytest.mark.parametrize("head_dim,n_heads,n_kv_heads,page,dtype", [
    (64, 4, 4, 16, torch.bfloat16), (64, 8, 2, 64, torch.float16), (96, 5, 5, 32, torch.float16),
    (96, 24, 4, 128, torch.bfloat16), (128, 32, 8, 64, torch.bfloat16), (128, 3, 3, 128, torch.float16),
    (128, 16, 1, 16, torch.bfloat16)])
@pytest.mark.parametrize("q_len", [1, 3])
def test_shared_prefix(head_dim, n_heads, n_kv_heads, page, dtype, q_len):
    lens = [700 + 3, 700 + 130, 701 + q_len, 700 + 1, 1200, 700 + 64]
    n_new = [1 + i % q_len for i in range(len(lens))]
    groups, shared = [(0, 6)], [700]
    cache, slots, gen = build(lens, shared, groups, page, n_kv_heads, head_dim, dtype, seed=head_dim + page + q_len)
    run(cache, slots, gen, n_heads, q_len, n_new, groups, shared)
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("lens", [[0], [1], [1, 0, 2, 15, 16, 17], [127, 128, 129, 255, 256, 257], [31, 33, 63, 65, 5000]])
def test_lengths_without_sharing(page, lens):
    cache, slots, gen = build(lens, [], [], page, 2, 64, torch.bfloat16, seed=len(lens) + page)
    run(cache, slots, gen, 4, 1)
    run(cache, slots, gen, 4, 4)          # more new tokens than some sequences have: their rows are empty
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("n_new,q_len", [([0, 0, 0], 2), ([2, 0, 1], 2), ([5, 9, 16], 16)])
def test_ragged_new_tokens(n_new, q_len):
    lens = [300, 290, 333]
    groups, shared = [(0, 3)], [280]
    cache, slots, gen = build(lens, shared, groups, 16, 2, 128, torch.bfloat16, seed=q_len)
    run(cache, slots, gen, 8, q_len, n_new, groups, shared)


def test_new_tokens_that_reach_into_the_prefix():
    """The last tokens of the prefix are the queries themselves: every row has its own end inside shared pages."""
    lens = [512, 512, 640]
    groups, shared = [(0, 3)], [512]
    cache, slots, gen = build(lens, shared, groups, 64, 2, 64, torch.bfloat16, seed=1)
    run(cache, slots, gen, 4, 32, [32, 7, 1], groups, shared)


def test_groups_of_all_sizes_and_requests_outside_them():
    lens = [900, 910, 950, 130, 140, 20, 2000, 2001, 2002, 2003, 2100, 77]
    groups, shared = [(0, 3), (3, 5), (5, 5), (5, 6), (6, 11)], [880, 128, 500, 10, 1999]
    cache, slots, gen = build(lens, shared, groups, 32, 2, 96, torch.bfloat16, seed=4)
    run(cache, slots, gen, 6, 2, [2] * 12, groups, shared)
    groups, shared = [(1, 3), (3, 5)], [880, 128]
    run(cache, slots, gen, 6, 2, [2] * 12, groups, shared)


def test_a_declared_prefix_longer_than_its_members_is_cut():
    lens = [130, 300, 260]
    groups, shared = [(0, 3)], [100000]
    cache, slots, gen = build(lens, [130], groups, 16, 1, 64, torch.bfloat16, seed=8)
    run(cache, slots, gen, 2, 1, None, groups, shared)
    run(cache, slots, gen, 2, 1, None, groups, [0])
    run(cache, slots, gen, 2, 1, None, groups, [-5])


def test_unused_requests():
    lens = [400, 420, 390, 500]
    groups, shared = [(0, 4)], [384]
    cache, slots, gen = build(lens, shared, groups, 64, 2, 128, torch.bfloat16, seed=3)
    for off in ([0], [3], [0, 1, 2], [0, 1, 2, 3]):
        s = [-1 if i in off else x for i, x in enumerate(slots)]
        run(cache, s, gen, 4, 2, [1, 2, 1, 2], groups, shared)


@pytest.mark.parametrize("B,q_len,n_heads,n_kv_heads", [(33, 4, 8, 2), (65, 1, 16, 4), (300, 1, 4, 4), (9, 31, 4, 1), (129, 2, 2, 2),
                                                        (1024, 1, 1, 1)])
def test_many_rows(B, q_len, n_heads, n_kv_heads):
    """Row counts around and past one and two tiles of 128."""
    r = random.Random(B)
    lens = [1000 + r.randint(q_len, 200) for _ in range(B)]
    groups, shared = [(0, B)], [1000]
    cache, slots, gen = build(lens, shared, groups, 32, n_kv_heads, 64, torch.bfloat16, seed=B)
    run(cache, slots, gen, n_heads, q_len, [r.randint(0, q_len) for _ in range(B)], groups, shared)


def test_long_sequences():
    lens = [30000, 30001, 17]
    groups, shared = [(0, 2)], [29990]
    cache, slots, gen = build(lens, shared, groups, 64, 1, 128, torch.bfloat16, seed=6)
    run(cache, slots, gen, 4, 1, None, groups, shared)
    run(cache, slots, gen, 4, 1)


def test_large_logits_and_scale():
    """Logits of a few hundred: the maximum moves between tiles and single keys dominate.  The rows' products add
    up to hundreds, so the logits' error allowance grows with them: keys are small integers here, which makes
    every product and sum exact."""
    lens = [1500, 1400]
    cache, slots, gen = build(lens, [], [], 32, 2, 64, torch.bfloat16, seed=12, poison=False)
    cache.pool[0] = torch.randint(-2, 3, cache.pool[0].shape, generator=gen, device="cuda").bfloat16()
    Q = torch.randint(-4, 5, (2, 4, 2, 64), generator=gen, device="cuda").bfloat16()
    O = torch.empty_like(Q)
    cache.attend(0, Q, O, u32(slots), None, None, None, 1.0)
    want, A = attention(cache, 0, Q, slots, [2, 2], 1.0)
    check_attention(O, want, A, 1500, 6.0)


def test_second_layer_and_its_planes():
    lens = [100, 260]
    cache, slots, gen = build(lens, [], [], 64, 2, 64, torch.float16, seed=2, n_layers=3)
    for layer in (2, 1, 0):
        run(cache, slots, gen, 2, 1, layer=layer)


def test_offsets_past_32_bits():
    """Pages whose byte offsets in a plane exceed 2^32."""
    n_pages = (1 << 32) // (8 * 128 * 128 * 2) + 64
    cache = serve.PagedCache(1, n_pages, 8, 128, 128, 2, 8)
    gen = torch.Generator(device="cuda").manual_seed(0)
    last = list(range(n_pages - 6, n_pages))
    cache.table[0, :6] = u32(last[::-1])
    cache.table[1, :6] = u32(last[::-1])
    cache.lens.copy_(u32([700, 650]))
    cache.refs[n_pages - 6:] = 2
    cache.pool[:, n_pages - 6:] = torch.randn((2, 6, 8, 128, 128), generator=gen, device="cuda").bfloat16()
    run(cache, [0, 1], gen, 32, 1, None, [(0, 2)], [640])
    run(cache, [1, 0], gen, 32, 1)


def test_faulty_slots_pages_lengths_and_groups():
    """Device data that breaks the rules is reported and stays in bounds; sound requests keep their results."""
    lens = [200, 210, 220, 230]
    cache, slots, gen = build(lens, [], [], 16, 2, 64, torch.bfloat16, seed=7, spare_slots=0)
    Q = torch.randn((4, 2, 1, 64), generator=gen, device="cuda").bfloat16()
    want, A = attention(cache, 0, Q, slots, [1] * 4)

    def bad(change, keep, n_new=None, start=None, shared=None, s=None):
        table, length = cache.table.clone(), cache.lens.clone()
        change()
        O = torch.empty_like(Q)
        cache.attend(0, Q, O, u32(slots if s is None else s), n_new, start, shared)
        assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
        if keep:
            check_attention(O[keep], want[keep], A[keep], 230, 6.0)
        cache.table.copy_(table)
        cache.lens.copy_(length)

    def set_table(s, k, v):
        cache.table[slots[s], k] = v

    def set_len(s, v):
        cache.lens[slots[s]] = v

    nothing = lambda: None  # noqa: E731
    bad(lambda: set_table(1, 3, -1), [0, 2, 3])
    bad(lambda: set_table(1, 3, cache.n_pages), [0, 2, 3])
    bad(lambda: set_table(1, 0, 2 ** 31 - 1), [0, 2, 3])
    bad(lambda: set_len(2, -4), [0, 1, 3])
    bad(lambda: set_len(2, 2 ** 30), [0, 1, 3])
    bad(nothing, [1, 2, 3], s=[4] + slots[1:])
    bad(nothing, [0, 1, 2], n_new=u32([1, 1, 1, 2]))
    bad(nothing, [0, 1, 2], n_new=u32([1, 1, 1, -1]))
    bad(nothing, [0, 1, 2, 3], start=u32([2, 1, 9]), shared=u32([0, 0]))
    bad(nothing, [0, 1, 2, 3], start=u32([-3, 1, 4]), shared=u32([0, 0]))


def test_repeats_are_bit_identical():
    lens = [3000 + 37 * i for i in range(20)]
    groups, shared = [(0, 20)], [3000]
    cache, slots, gen = build(lens, shared, groups, 64, 4, 128, torch.bfloat16, seed=5)
    Q = torch.randn((20, 16, 1, 128), generator=gen, device="cuda").bfloat16()
    outs = []
    for _ in range(6):
        O = torch.empty_like(Q)
        cache.attend(0, Q, O, u32(slots), None, u32([0, 20]), u32(shared))
        outs.append(O)
    for O in outs[1:]:
        assert torch.equal(O.view(torch.int16), outs[0].view(torch.int16))


def test_refusals():
    cache, slots, gen = build([40, 50], [], [], 16, 2, 64, torch.bfloat16, seed=7)
    Q = torch.randn((2, 4, 1, 64), device="cuda").bfloat16()
    s, O = u32(slots), torch.empty_like(Q)
    for args in ((Q.half(), O, s), (Q, O[:1], s), (Q, O, s.long()), (Q.transpose(0, 1), O, s), (Q, O, s[:1]),
                 (Q, O, s, u32([1])), (Q, O, s, None, u32([0, 2])), (Q, O, s, None, None, u32([3]))):
        with pytest.raises(ValueError):
            cache.attend(0, *args)
    with pytest.raises(wise.WiseError):
        cache.attend(1, Q, O, s)
    with pytest.raises(wise.WiseError):
        cache.attend(0, Q[:, :3].contiguous(), O[:, :3].contiguous(), s)
    with pytest.raises(wise.WiseError):
        big = torch.zeros((2, 4, 65, 64), dtype=torch.bfloat16, device="cuda")
        cache.attend(0, big, torch.empty_like(big), s)
