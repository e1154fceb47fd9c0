"""Writing to caches in 8 or 4 bits and reading back, against tables of all numbers in fp64: bit for bit."""
import random

import pytest
import torch

from paper_2609_27373_gb300 import serve, wise
from quant_helpers import build, stored
from serve_helpers import u32

pytestmark = pytest.mark.gpu


def new_cache(bits, page, kv, dim, dtype, n_slots=4, max_pages=8, n_pages=32, n_layers=1):
    c = serve.PagedCache(n_layers, n_pages, kv, page, dim, n_slots, max_pages, dtype, bits=bits)
    if bits == 16:
        c.pool.fill_(float("nan"))
    else:
        c.pool.random_(0, 256)
    return c


def rows(c, slot, n, layer=0):
    """The first n positions of a sequence as [2, kv, n, dim]."""
    out = torch.full((2, 1, c.n_kv_heads, n, c.head_dim), float("nan"), dtype=c.dtype, device="cuda")
    c.read(layer, out[0], out[1], u32([slot]))
    return out[:, 0]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("page,dim,kv,dtype", [
    (16, 64, 4, torch.bfloat16), (32, 96, 5, torch.float16), (64, 128, 2, torch.bfloat16), (128, 128, 1, torch.float16),
    (16, 128, 3, torch.float16), (128, 64, 2, torch.bfloat16), (16, 96, 1, torch.bfloat16)])
def test_sequences_written_in_pieces(bits, page, dim, kv, dtype):
    """Single tokens, drafts and prompts after one another; every token keeps its value and is where it was put."""
    r = random.Random(page + dim + bits)
    c = new_cache(bits, page, kv, dim, dtype, n_slots=3, max_pages=-(-400 // page), n_pages=3 * -(-400 // page))
    gen = torch.Generator(device="cuda").manual_seed(page * dim)
    said = [torch.empty((2, kv, 0, dim), dtype=torch.float64, device="cuda") for _ in range(3)]
    for most in (1, 1, 3, 40, 1, 1, 17, 90, 2, 1, 130, 1, 31):
        order = r.sample(range(3), 3)
        n = [r.randint(0, most) for _ in order]
        n[r.randrange(3)] = most
        granted = c.extend(u32(order), u32(n))
        x = (torch.randn((2, 3, kv, most, dim), generator=gen, device="cuda") *
             torch.exp(2 * torch.randn((2, 3, kv, most, 1), generator=gen, device="cuda"))).to(dtype)
        c.write(0, u32(order), granted, x[0], x[1])
        for i, slot in enumerate(order):
            said[slot] = torch.cat([said[slot], stored(x[:, i, :, :n[i]], bits)], 2)
    for slot in range(3):
        n = said[slot].shape[2]
        assert torch.equal(rows(c, slot, n).double(), said[slot])
    # Spans of each, rows that do not exist, and an unused entry.
    first, count = [3, 0, 5, 7], [9, 33, 40, 0]
    K = torch.full((4, kv, 40, dim), float("nan"), dtype=dtype, device="cuda")
    V = K.clone()
    c.read(0, K, V, u32([2, 0, -1, 1]), u32(first), u32(count))
    for i, slot in enumerate([2, 0, None, 1]):
        want = torch.zeros((2, kv, 40, dim), dtype=torch.float64, device="cuda")
        if slot is not None:
            part = said[slot][:, :, first[i]:first[i] + count[i]]
            want[:, :, :part.shape[2]] = part
        assert torch.equal(torch.stack([K[i], V[i]]).double(), want)
    n = said[1].shape[2]
    K = torch.full((1, kv, 50, dim), float("nan"), dtype=dtype, device="cuda")
    V = K.clone()
    c.read(0, K, V, u32([1]), u32([n - 7]))                      # ends inside the rows
    assert torch.equal(torch.stack([K[0, :, :7], V[0, :, :7]]).double(), said[1][:, :, -7:])
    assert not K[0, :, 7:].any() and not V[0, :, 7:].any()
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_sizes_and_ties(bits, dtype):
    """Scales from the smallest to the largest, quotients half way between two codes, zeros, the type's extremes."""
    dim, kv = 64, 1
    scales = [m / 8 * 2.0 ** e for e in range(-14, 14) for m in range(8, 16) if m / 8 * 2.0 ** e <= 10240]
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]
    groups = []
    for s in scales + [m * 2.0 ** -17 for m in range(8)]:
        g = [m * s for m in mids] + [-m * s for m in mids]
        g[15] = -6.0 * s
        groups.append(g)
        groups.append([x * 1.01 for x in g])
    for k in range(-18, 9):
        for top in (448.0, 449.0, 450.0, 400.0, 256.0):
            q = [top, 0.0, -17.0, 17.0, 1.0625, 0.0009765625, 0.0029296875, 440.0, -432.0, 2.0 ** -10, 2.0 ** -9, 12.5, 13.5,
                 0.02, -0.017578125, 224.0]
            groups.append([x * 2.0 ** k for x in q])
    top = float(torch.finfo(dtype).max)
    groups += [[0.0] * 16, [top, -top] + [1.0] * 14, [2.0 ** -24] * 16, [float(torch.finfo(dtype).tiny)] * 16]
    while len(groups) % 4:
        groups.append([0.0] * 16)
    x = torch.tensor(groups, dtype=torch.float64).to(dtype).cuda()
    x = torch.where(torch.isinf(x), torch.full_like(x, top), x).reshape(1, kv, -1, dim)
    n = x.shape[2]
    c = new_cache(bits, 16, kv, dim, dtype, n_slots=1, max_pages=-(-n // 16), n_pages=-(-n // 16))
    c.write(0, u32([0]), c.extend(u32([0]), u32([n])), x, -x)
    got, want = rows(c, 0, n).double(), stored(x[0], bits)
    assert torch.equal(got[0], want) and torch.equal(got[1], -want)


@pytest.mark.parametrize("bits,limit", [(4, 61440.0), (8, 57344.0)])
def test_infinities(bits, limit):
    x = torch.ones((1, 1, 1, 64), dtype=torch.bfloat16, device="cuda")
    x[..., 3], x[..., 20] = float("inf"), -float("inf")
    c = new_cache(bits, 16, 1, 64, torch.bfloat16)
    c.write(0, u32([0]), c.extend(u32([0]), u32([1])), x, x)
    got = rows(c, 0, 1)[:, 0, 0].double().tolist()
    others = stored(x[..., 32:], bits).flatten().tolist()
    for v in got:
        assert v[3] == limit and v[20] == -limit and v[32:] == others


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("page,dim", [(16, 96), (64, 128), (128, 64)])
def test_forks_copies_and_compaction(bits, page, dim):
    kv, layers = 3, 2
    c = new_cache(bits, page, kv, dim, torch.bfloat16, n_slots=6, max_pages=6, n_pages=40, n_layers=layers)
    gen = torch.Generator(device="cuda").manual_seed(7)
    said = {}

    def grow(slots, n):
        granted = c.extend(u32(slots), u32([n] * len(slots)))
        assert granted.tolist() == [n] * len(slots)
        for layer in range(layers):
            x = torch.randn((2, len(slots), kv, n, dim), generator=gen, device="cuda").to(torch.bfloat16)
            c.write(layer, u32(slots), granted, x[0], x[1])
            for i, s in enumerate(slots):
                old = said.get((s, layer), torch.empty((2, kv, 0, dim), dtype=torch.float64, device="cuda"))
                said[s, layer] = torch.cat([old, stored(x[:, i], bits)], 2)

    def check(slots):
        for s in slots:
            for layer in range(layers):
                assert torch.equal(rows(c, s, said[s, layer].shape[2], layer).double(), said[s, layer]), (s, layer)

    grow([0, 5], 2 * page + 5)
    c.fork(u32([0, 0]), u32([1, 3]))
    for layer in range(layers):
        said[1, layer] = said[3, layer] = said[0, layer]
    grow([1, 3], 1)                       # each gets a copy of the last page
    grow([0], 3)
    check([0, 1, 3, 5])
    c.drop(u32([5, 3]), u32([1 << 20, page + 2]))
    for layer in range(layers):
        said[3, layer] = said[3, layer][:, :, :-(page + 2)]
    remap, live = c.compact()
    assert int(live) < 40 and wise.wise_get_status() == wise.WISE_OK
    check([0, 1, 3])
    grow([3, 0], page)
    check([0, 1, 3])


@pytest.mark.parametrize("bits", [4, 8])
def test_faults_leave_rows_out(bits):
    page, dim, kv = 16, 64, 2
    c = new_cache(bits, page, kv, dim, torch.bfloat16, n_slots=5, max_pages=4, n_pages=20)
    granted = c.extend(u32([0, 1, 2, 3]), u32([20, 20, 20, 20]))
    ones = torch.ones((4, kv, 20, dim), dtype=torch.bfloat16, device="cuda")
    c.write(0, u32([0, 1, 2, 3]), granted, ones, ones)
    c.fork(u32([3]), u32([4]))
    c.table[1, 1] = 20                                           # no page
    before = c.pool.clone()
    twos = ones * 2
    c.write(0, u32([2, 1, 2, 4]), u32([5, 4, 5, 5]), twos[:, :, :5].contiguous(), twos[:, :, :5].contiguous())
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE     # listed twice, page 20, a page of two holders
    assert torch.equal(c.pool, before)
    for slots, new in (([7], [1]), ([0], [21]), ([0], [-1])):
        c.write(0, u32(slots), u32(new), twos[:1, :, :20].contiguous(), twos[:1, :, :20].contiguous())
        assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
        assert torch.equal(c.pool, before)
    c.write(0, u32([-1, -1]), None, twos[:2], twos[:2])
    assert wise.wise_get_status() == wise.WISE_OK and torch.equal(c.pool, before)
    # Reading: the page without a sound id, and faulty entries, become zeros.
    K = torch.full((6, kv, 20, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    V = K.clone()
    c.read(0, K, V, u32([1, 0, 9, 0, 0, 0]), u32([0, 2, 0, -1, 0, 65]), u32([20, 18, 20, 20, 21, 1]))
    assert wise.wise_get_status() == wise.WISE_ERR_BAD_CACHE
    one = float(stored(ones, bits)[0, 0, 0, 0])
    for x in (K, V):
        assert (x[0, :, :16] == one).all() and not x[0, :, 16:].any()
        assert (x[1, :, :18] == one).all() and not x[1, :, 18:].any()
        assert not x[2:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_reading_16_bits(dtype):
    c = new_cache(16, 32, 3, 96, dtype, n_layers=2)
    x = torch.randn((2, 2, 3, 75, 96), device="cuda").to(dtype)
    granted = c.extend(u32([2, 0]), u32([75, 41]))
    c.write(1, u32([2, 0]), granted, x[0], x[1])
    got = rows(c, 2, 75, 1)
    assert torch.equal(got, x[:, 0])
    assert torch.equal(rows(c, 0, 41, 1), x[:, 1, :, :41])


def test_large_batches_and_offsets():
    """More requests than resident warps, and pages past 2^31 bytes into the pool."""
    page, dim, kv = 128, 128, 8
    c = serve.PagedCache(1, 18000, kv, page, dim, 2000, 1, torch.bfloat16, bits=4)
    assert c.pool.numel() > 2 ** 31
    order = torch.randperm(2000, device="cuda").int()
    c.table.copy_((17999 - torch.arange(2000, device="cuda")).int()[:, None])
    c.lens.fill_(3)
    c.refs[-2000:] = 1
    x = torch.randn((2, 2000, kv, 3, dim), device="cuda").to(torch.bfloat16)
    c.write(0, order, None, x[0], x[1])
    got = torch.empty_like(x)
    c.read(0, got[0], got[1], order)
    assert torch.equal(got.double(), stored(x, 4))
    assert wise.wise_get_status() == wise.WISE_OK


@pytest.mark.parametrize("bits", [4, 8])
def test_captured(bits):
    c, twin, slots, gen = build(bits, [50, 70], 16, 2, 64, torch.bfloat16, seed=3)
    x = torch.randn((2, 2, 2, 4, 64), generator=gen, device="cuda").to(torch.bfloat16)
    out, new = torch.empty_like(x), u32([4, 4])
    s, first = u32(slots), u32([46, 66])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.write(0, s, new, x[0], x[1])
        c.read(0, out[0], out[1], s, first)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out.double(), stored(x, bits))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.write(0, s, new, x[0], x[1])
        c.read(0, out[0], out[1], s, first)
    x.mul_(-3)
    new.copy_(u32([4, 2]))
    first.copy_(u32([46, 68]))
    g.replay()
    want = stored(x, bits)
    assert torch.equal(out[:, 0].double(), want[:, 0])
    assert torch.equal(out[:, 1, :, :2].double(), want[:, 1, :, :2]) and not out[:, 1, :, 2:].any()
