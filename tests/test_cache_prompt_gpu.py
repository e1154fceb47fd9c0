"""Prompts taken into the cache: long extends and writes (integers and copied rows: every comparison is exact)."""
import random

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import ListCache, u32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,head_dim,n_kv_heads,n_new", [
    (16, 128, 2, [5000, 0, 4999, 16]), (64, 96, 3, [4096, 2047, 1, 3333]), (128, 64, 1, [30000, 127, 129]),
    (32, 128, 8, [2500])])
def test_prompts(page, head_dim, n_kv_heads, n_new):
    """More rows than the blocks that stay resident take at once, in unlike lengths, into pages in a mixed order."""
    r = random.Random(page)
    B, q_len = len(n_new), max(n_new)
    max_pages = -(-q_len // page) + 1
    n_pages = sum(-(-n // page) for n in n_new) + 40
    cache = serve.PagedCache(2, n_pages, n_kv_heads, page, head_dim, B + 2, max_pages)
    model = ListCache(n_pages, page, B + 2, max_pages)
    taken = r.sample(range(n_pages), 30)
    for g in taken:
        model.refs[g] = 1
    cache.refs.copy_(u32(model.refs))
    slots = r.sample(range(B + 2), B)
    want, _ = model.extend(slots, n_new)
    granted = cache.extend(u32(slots), u32(n_new))
    assert granted.tolist() == want == n_new
    model.matches(cache)
    pool = cache.pool.normal_().clone()
    gen = torch.Generator(device="cuda").manual_seed(page)
    for layer in (1, 0):
        x = [torch.randn((B, n_kv_heads, q_len, head_dim), generator=gen, device="cuda").bfloat16() for _ in range(2)]
        cache.write(layer, u32(slots), granted, *x)
        for b, s in enumerate(slots):
            at = torch.arange(n_new[b], device="cuda")
            rows = cache.table[s].long()[at // page]
            for k in range(2):
                pool[2 * layer + k, rows, :, at % page] = x[k][b, :, :n_new[b]].transpose(0, 1)
    assert torch.equal(cache.pool.view(torch.int16), pool.view(torch.int16))
    assert wise.wise_get_status() == wise.WISE_OK
