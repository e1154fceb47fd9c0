"""What a cache in 8 or 4 bits holds, by looking every number up in fp64, and caches with a 16-bit twin."""
import random

import torch

from paper_2609_27373_gb300 import serve
from serve_helpers import u32

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def small_floats(lowest, most):
    """0 and all numbers with 3 mantissa bits up to `most`; below 2^lowest they are 2^(lowest - 3) apart."""
    out = [m * 2.0 ** (lowest - 3) for m in range(8)]
    e = lowest
    while out[-1] < most:
        out += [(1 + m / 8) * 2.0 ** e for m in range(8)]
        e += 1
    return [x for x in out if x <= most]


def nearest(table, y):
    t = torch.tensor(table, dtype=torch.float64, device=y.device)
    mid = (t[1:] + t[:-1]) / 2
    i = torch.searchsorted(mid, y.contiguous())
    tie = y == mid[torch.clamp(i, max=len(table) - 2)]
    return t[torch.where(tie & (i % 2 == 1), i + 1, i)]


def stored(x, bits):
    """The values that x [..., head_dim] is stored as, fp64."""
    g = x.double().reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    a = g.abs().amax(-1, True)
    if bits == 4:
        s = nearest(small_floats(-14, 10240.0), a / torch.full_like(a, 6.0))
        q = nearest(E2M1, torch.where(s > 0, g.abs() / torch.where(s > 0, s, 1.0), 0.0))
    else:
        k = torch.full_like(a, -15.0)
        for j in range(-15, 7):
            k = torch.where(a > 448.0 * 2.0 ** j, j + 1.0, k)
        s = torch.exp2(k)
        q = nearest(small_floats(-6, 448.0), g.abs() / s)
    return (torch.sign(g) * q * s).reshape(x.shape)


class Twin:
    """The cache `shadow` of 16 bits with the values that `cache` stands for, for serve_helpers.attention."""

    def __init__(self, cache, pool):
        self.pool, self.table, self.lens = pool, cache.table, cache.lens
        self.page, self.n_kv_heads = cache.page, cache.n_kv_heads


def build(bits, lens, page, n_kv_heads, head_dim, dtype, seed, groups=(), shared=(), n_layers=1, spread=1.0):
    """A cache whose requests have the given lengths, its twin, the requests' slots and a generator.  The requests of
    groups[g] = (start, end) share the pages of their first shared[g] tokens.  Bytes that hold no token are random."""
    r = random.Random(seed)
    B = len(lens)
    slots = r.sample(range(B + 2), B)
    n_pages = sum(-(-n // page) for n in lens) + 3
    ids = r.sample(range(n_pages), n_pages)
    max_pages = max([-(-n // page) for n in lens] + [1]) + 1
    table = [[r.randrange(n_pages) for _ in range(max_pages)] for _ in range(B + 2)]  # unused entries mean nothing
    length, refs, common = [0] * (B + 2), [0] * n_pages, {}
    for (a, b), tokens in zip(groups, shared):
        whole = min([lens[i] for i in range(a, b)] + [tokens]) // page
        pages = [ids.pop() for _ in range(whole)]
        for i in range(a, b):
            common[i] = pages
    for i, n in enumerate(lens):
        row = list(common.get(i, []))
        row += [ids.pop() for _ in range(-(-n // page) - len(row))]
        table[slots[i]][:len(row)] = row
        length[slots[i]] = n
        for g in row:
            refs[g] += 1
    gen = torch.Generator(device="cuda").manual_seed(seed)
    values = (torch.randn((2 * n_layers, n_pages, n_kv_heads, page, head_dim), generator=gen, device="cuda") * spread).to(dtype)
    whole = serve.PagedCache(n_layers, n_pages, n_kv_heads, page, head_dim, n_pages, 1, dtype, bits=bits)
    whole.pool.copy_(torch.randint(0, 256, whole.pool.shape, generator=gen, device="cuda", dtype=torch.uint8))
    # Each page is written as a sequence of its own, as many tokens as it holds.
    held = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    tab, ln = u32(table), u32(length)
    for s in range(B + 2):
        at = torch.arange(length[s], device="cuda")
        held.scatter_reduce_(0, tab[s].long()[at // page], (at % page + 1).int(), "amax")
    whole.table.copy_(torch.arange(n_pages, dtype=torch.int32, device="cuda")[:, None])
    whole.lens.copy_(held)
    whole.refs.fill_(1)
    for layer in range(n_layers):
        whole.write(layer, torch.arange(n_pages, dtype=torch.int32, device="cuda"), held, values[2 * layer].contiguous(),
                    values[2 * layer + 1].contiguous())
    cache = serve.PagedCache.over(whole.pool, tab, ln, u32(refs), bits=bits, page=page, head_dim=head_dim, dtype=dtype)
    return cache, Twin(cache, stored(values, bits)), slots, gen


def check_attention(O, want, A, n_keys, vmax):
    """Bound of |O - want|, element by element, with u the unit roundoff of O's type (2^-8 for bf16, 2^-11 for fp16): the
    rounding of O, u |O|; the softmax numerators, rounded to fp16 (2^-11 each, in the sum of values and, where that is
    made of rounded ones, in their own sum), 2^-10 A; logits summed in fp32 over at most 128 products and the fast
    exponential, 2^-10 A for logits whose products add up to a few tens; numerators below fp16's normal range, which are
    held 2^7 higher against a sum of at least 1, 2^-32 each and as much again for their sum."""
    u = 2.0 ** -8 if O.dtype is torch.bfloat16 else 2.0 ** -11
    tol = u * want.abs() + 2.0 ** -9 * A + n_keys * 2.0 ** -31 * vmax + 1e-7
    got = O.double()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol
    assert float(over.max()) <= 0.0, f"worst excess {float(over.max()):.3e}, error {float((got - want).abs().max()):.3e}"
