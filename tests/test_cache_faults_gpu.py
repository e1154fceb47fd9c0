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
