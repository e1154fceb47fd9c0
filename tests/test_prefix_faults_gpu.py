"""Attention over caches with faulty pages."""
import pytest
import torch

from paper_2609_27373_gb300 import wise
from serve_helpers import attention, check_attention, u32
from test_prefix_attn_gpu import build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,q_len,n_heads,n_kv_heads,head_dim", [(5, 1, 4, 2, 64), (6, 3, 6, 3, 96), (100, 2, 8, 2, 128),
                                                                 (70, 4, 16, 4, 64)])
@pytest.mark.parametrize("page", [16, 128])
def test_requests_that_read_a_faulty_page_give_zero(B, q_len, n_heads, n_kv_heads, head_dim, page):
    """A faulty id in a request's own keys concerns that request; one in a shared prefix, read through the first
    active member's row, all of its group.  The other requests keep their results."""
    half = B // 2
    lens = [700 + 3 + q_len + (37 * i) % 400 for i in range(B)]
    groups, shared = [(0, half), (half, B)], [690, 512]
    cache, slots, gen = build(lens, shared, groups, page, n_kv_heads, head_dim, torch.bfloat16, seed=B + page)
    Q = torch.randn((B, n_heads, q_len, head_dim), generator=gen, device="cuda").bfloat16()
    start, pre = u32([0, half, B]), u32(shared)
    want, A = attention(cache, 0, Q, slots, [q_len] * B)

    def check(faults, concerned):
        table = cache.table.clone()
        for i, k, g in faults:
            cache.table[slots[i], k] = g
        O = torch.full_like(Q, float("nan"))
        cache.attend(0, Q, O, u32(slots), None, start, pre)
        assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
        cache.table.copy_(table)
        sound = [i for i in range(B) if i not in concerned]
        for i in concerned:
            assert not O[i].float().abs().max().item(), (faults, i)
        if sound:
            check_attention(O[sound], want[sound], A[sound], max(lens), 6.0)

    last = B - 1
    own = (lens[last] - 1) // page
    check([(last, own, -1)], [last])                                        # the last page of one request
    check([(1, (lens[1] - 1) // page, cache.n_pages), (last, own, 1 << 30)], [1, last])
    check([(0, 0, -1)], list(range(half)))                                  # the first page of the first group's prefix
    check([(half, 512 // page - 1, cache.n_pages)], list(range(half, B)))   # the last page of the second one's
    check([(0, 2, -5), (half, 1, -5)], list(range(B)))


def test_a_faulty_page_without_groups_and_over_many_segments():
    """One long sequence is split over many CTAs; the fault lies in one part of it."""
    lens = [40000, 300]
    cache, slots, gen = build(lens, [], [], 64, 1, 128, torch.float16, seed=3)
    Q = torch.randn((2, 4, 1, 128), generator=gen, device="cuda").half()
    want, A = attention(cache, 0, Q, slots, [1, 1])
    for k in (0, 311, 624):
        table = cache.table.clone()
        cache.table[slots[0], k] = -1
        O = torch.full_like(Q, float("nan"))
        cache.attend(0, Q, O, u32(slots))
        assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
        cache.table.copy_(table)
        assert not O[0].float().abs().max().item()
        check_attention(O[1:], want[1:], A[1:], 300, 6.0)
