"""Attention over the paged cache where a row's numerators differ by many orders of magnitude."""
import math

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from serve_helpers import u32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_million_keys_far_below_the_maximum(dtype):
    """One key has all but 2^-26 of every other one's weight, and there are 2^20 others, which together have 1.5 %.
    Enough requests read them that a segment is as long as a sequence.  Besides the roundings that check_attention
    allows for, a numerator may be off by half of fp16's smallest step, 2^-25, where the row's largest one is held as
    2^7 or more: 2^-32 a key."""
    n, B, page = 1 << 20, 320, 128
    cache = serve.PagedCache(1, n // page, 1, page, 64, B, n // page, dtype)
    cache.pool.zero_()
    cache.pool[0, 0, 0, 0, 0] = 4.5
    cache.pool[1] = 1.0
    cache.pool[1, 0, 0, 0] = 0.0
    cache.table.copy_(torch.arange(n // page, dtype=torch.int32, device="cuda").expand(B, -1))
    cache.lens.fill_(n)
    cache.refs.fill_(B)
    Q = torch.zeros((B, 1, 1, 64), dtype=dtype, device="cuda")
    Q[..., 0] = 4.0
    O = torch.empty_like(Q)
    cache.attend(0, Q, O, torch.arange(B, dtype=torch.int32, device="cuda"), None, None, None, 1.0)
    assert wise.wise_get_status() == wise.WISE_OK
    rest = (n - 1) * math.exp(-18.0)
    want = torch.full((B, 1, 1, 64), rest / (1 + rest), dtype=torch.float64, device="cuda")
    u = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -11
    tol = (2 * u + 2.0 ** -10) * float(want[0, 0, 0, 0]) + (0.0 if dtype is torch.bfloat16 else n * 2.0 ** -32)
    err = float((O.double() - want).abs().max())
    assert err <= tol, (err, tol, float(want[0, 0, 0, 0]))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rise", [2.0, 7.5, 8.5, 20.0])
def test_a_maximum_that_rises_from_tile_to_tile(dtype, rise):
    """Each tile of 128 keys has logits of `rise` bits more than the one before: numerators grow past the first
    maximum up to the threshold at which it moves, and must stay finite.  Keys and queries are powers of two and small
    integers, so the logits are exact up to fp32's rounding of their scaling."""
    tiles, page, D = 12, 128, 64
    cache = serve.PagedCache(1, tiles, 1, page, D, 1, tiles, dtype)
    cache.table[0] = torch.arange(tiles, dtype=torch.int32, device="cuda")
    cache.lens.fill_(tiles * page)
    cache.refs.fill_(1)
    cache.pool.zero_()
    for t in range(tiles):
        cache.pool[0, t, 0, :, 0] = t
    cache.pool[1] = torch.randn(cache.pool[1].shape, device="cuda").to(dtype)
    Q = torch.zeros((1, 1, 1, D), dtype=dtype, device="cuda")
    Q[..., 0] = 1.0
    O = torch.empty_like(Q)
    scale = rise * math.log(2.0)
    cache.attend(0, Q, O, u32([0]), None, None, None, scale)
    assert wise.wise_get_status() == wise.WISE_OK
    v = cache.pool[1, :, 0].reshape(-1, D).double()
    w = torch.softmax(torch.arange(tiles, device="cuda").double().repeat_interleave(page) * float(torch.tensor(scale)), 0)
    want, A = w @ v, w @ v.abs()
    u = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -11
    # The logits reach 240 bits, of which fp32 rounds 2^-17 away; ex2 and the sums add less.
    err = (O[0, 0, 0].double() - want).abs() - (u * want.abs() + (u + 2.0 ** -10) * A + 1e-7)
    assert torch.isfinite(O).all() and float(err.max()) <= 0.0
