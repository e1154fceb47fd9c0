"""Workloads of the quantised paged cache: storing keys and values in 8 or 4 bits, reading them back, and attention of a
batch over them.

Each workload can run in its plain form (elementary torch operations in 32 bits) or through the package; `own`
chooses.  Sizes are those of this package's configurations (4 heads of 64; 32 heads of 128 at 4K; 55 heads of 96;
32 query heads over 8 key heads of 128 at 32K) with generic batches, lengths and page sizes.

Groups of 16 neighbouring values of a row share a scale s.  4 bits: s is the nearest number of 5 exponent and 3 mantissa
bits to a sixth of the group's largest size, the value s times the nearest of 0, 0.5, 1, 1.5, 2, 3, 4 and 6 with a sign.
8 bits: s is the smallest power of two with which the largest size is at most 448, the value s times the nearest
number of 4 exponent and 3 mantissa bits.  Ties go to the even code.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
KEPT = 20  # older tokens that a stored case reads back beside the new ones


def listed():
    return [
        # A token each for two short sequences: one layer of a decoding step, where only latency counts.
        dict(name="store_small", kind="store", bits=4, dtype="bf16", kv_heads=4, head_dim=64, page=16, batch=2,
             before=40, q_len=1),
        # Ragged drafts of up to 5 tokens at the ends of a full batch of sequences.
        dict(name="store_drafts", kind="store", bits=8, dtype="bf16", kv_heads=8, head_dim=128, page=64, batch=256,
             before=700, q_len=5),
        # Prompts of odd lengths that continue sequences in the middle of a page, 55 heads of 96, fp16.
        dict(name="store_odd_d96", kind="store", bits=4, dtype="fp16", kv_heads=55, head_dim=96, page=32, batch=5,
             before=77, q_len=1501),
        # Two long prompts, grouped heads.
        dict(name="store_32k", kind="store", bits=4, dtype="bf16", kv_heads=8, head_dim=128, page=64, batch=2,
             before=0, q_len=32768),
        # The last tokens of a short sequence.
        dict(name="read_small", kind="read", bits=4, dtype="bf16", kv_heads=4, head_dim=64, page=16, batch=1,
             length=60, rows=40),
        # Odd spans out of sequences in 8 bits, 55 heads of 96, fp16.
        dict(name="read_odd_d96", kind="read", bits=8, dtype="fp16", kv_heads=55, head_dim=96, page=32, batch=7,
             length=1500, rows=777),
        # Two whole documents, for a pass that wants dense keys and values.
        dict(name="read_32k", kind="read", bits=4, dtype="bf16", kv_heads=8, head_dim=128, page=64, batch=2,
             length=32768, rows=32768),
        # One prompt sampled twice: a handful of cached tokens, where only latency counts.
        dict(name="attend_small", kind="attend", bits=4, dtype="bf16", heads=4, kv_heads=4, head_dim=64, page=16,
             groups=1, batch=2, prefix=512, suffix=40, q_len=1),
        # 16 unrelated sequences, every query head with its own keys, 8 bits.
        dict(name="attend_4k_8bit", kind="attend", bits=8, dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=64,
             groups=0, batch=16, prefix=16000, suffix=500, q_len=1),
        # Ragged drafts of up to 3 tokens, 55 heads of 96, a prefix that ends inside a page, fp16.
        dict(name="attend_odd_d96", kind="attend", bits=4, dtype="fp16", heads=55, kv_heads=55, head_dim=96, page=32,
             groups=1, batch=7, prefix=4001, suffix=777, q_len=3),
        # 32 long conversations that share nothing, grouped heads: the cache's bytes are all that counts.
        dict(name="attend_long", kind="attend", bits=4, dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=64,
             groups=0, batch=32, prefix=32768, suffix=8192, q_len=1),
        # A long document asked 64 questions: 32K shared tokens, grouped heads.
        dict(name="attend_32k_shared", kind="attend", bits=4, dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=64,
             groups=1, batch=64, prefix=32768, suffix=1024, q_len=1),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attend", "attend", "attend", "store", "read"])
    c = dict(kind=kind, bits=rng.choice([4, 4, 8]), dtype=rng.choice(["bf16", "bf16", "fp16"]))
    heads, kv_heads, head_dim = rng.choice([(4, 4, 64), (32, 32, 128), (55, 55, 96), (32, 8, 128), (8, 2, 64), (24, 4, 96)])
    c.update(kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]))
    if kind == "attend":
        c.update(heads=heads, groups=rng.choice([0, 0, 1, 1, 2, 3]), batch=log(1, 256), prefix=log(1, 65536),
                 suffix=log(1, 16384), q_len=rng.choice([1, 1, 2, 3, 4, 5, 8]))
        c["groups"] = min(c["groups"], c["batch"])
        c["suffix"] = max(c["suffix"], c["q_len"])
        while work(c)["flops"] > 3e10 or work(c)["bytes"] > 6e8 or _plain_values(c) > 6e8:
            c["batch"], c["prefix"] = max(c["groups"], 1, c["batch"] * 2 // 3), max(1, c["prefix"] * 3 // 4)
            c["suffix"] = max(c["q_len"], c["suffix"] * 3 // 4)
        return c
    if kind == "store":
        c.update(batch=log(1, 256), before=rng.choice([0, log(1, 2048)]), q_len=log(1, 32768))
        while work(c)["bytes"] > 6e8 or c["batch"] * (c["before"] + c["q_len"]) * kv_heads * head_dim > 1.5e8:
            c["batch"], c["q_len"] = max(1, c["batch"] * 2 // 3), max(1, c["q_len"] * 2 // 3)
            c["before"] = c["before"] * 3 // 4
        return c
    c.update(batch=log(1, 64), length=log(1, 32768))
    c["rows"] = max(1, int(c["length"] * rng.choice([1.0, rng.uniform(0.05, 1.0)])))
    while work(c)["bytes"] > 6e8 or c["batch"] * c["length"] * kv_heads * head_dim > 1.5e8:
        c["batch"], c["length"] = max(1, c["batch"] * 2 // 3), max(1, c["length"] * 3 // 4)
        c["rows"] = min(c["rows"], c["length"])
    return c


# ------------------------------------------------------------ the plain form
def _stored(x, bits):
    """The values that x [..., multiple of 16] is stored as, in 32 bits."""
    g = x.float().reshape(*x.shape[:-1], -1, 16)
    a = g.abs().amax(-1, True)
    if bits == 4:
        t = torch.clamp(a / torch.full_like(a, 6.0), max=10240.0)
        step = torch.exp2(torch.clamp(torch.frexp(t)[1] - 1, min=-14).float() - 3.0)  # of 4 significant bits
        s = torch.clamp(torch.round(t / step) * step, max=10240.0)
        y = torch.clamp(torch.where(s > 0, g / s, 0.0), -6.0, 6.0)
        size = y.abs()
        step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
        v = torch.round(y / step) * step * s
    else:
        m, e = torch.frexp(a)  # a = m 2^e with m in [0.5, 1); 448 = 0.875 * 2^9
        k = torch.clamp(e - 9 + (m > 0.875).int(), -15, 7).float()
        y = torch.clamp(g * torch.exp2(-k), -448.0, 448.0)
        step = torch.exp2(torch.clamp(torch.frexp(y)[1] - 1, min=-6).float() - 3.0)
        v = torch.round(y / step) * step * torch.exp2(k)
    return v.reshape(x.shape)


def _plain_write(s):
    """pool[...] at the new tokens' places = what K and V are stored as."""
    P, slots, new = s["case"]["page"], s["slots"].long(), s["new"]
    at = torch.nonzero(torch.arange(s["K"].shape[2], device="cuda") < new[:, None])
    pos = s["lens"][slots[at[:, 0]]] - new[at[:, 0]] + at[:, 1]
    to = s["table"][slots[at[:, 0]], (pos // P).long()].long()
    for plane, x in enumerate((s["K"], s["V"])):
        s["pool"][plane, to, :, (pos % P).long()] = _stored(x[at[:, 0], :, at[:, 1]], s["case"]["bits"]).to(x.dtype)


def _plain_read(s):
    P, (B, KV, rows, D) = s["case"]["page"], s["outK"].shape
    slots = s["slots"].long()
    i = torch.arange(rows, device="cuda")
    pos = s["first"][:, None] + i
    there = (i < s["count"][:, None]) & (pos < s["lens"][slots][:, None])
    pos = torch.where(there, pos, 0)
    page = s["table"][slots[:, None], (pos // P).long()].long()
    page = torch.where(there, page, 0)
    for plane, out in enumerate((s["outK"], s["outV"])):
        x = s["pool"][plane, page, :, (pos % P).long()]  # [B, rows, KV, D]
        out.copy_(torch.where(there[:, :, None, None], x, 0.0).permute(0, 2, 1, 3))
    return dict(K=s["outK"], V=s["outV"])


# -------------------------------------------------------- caches in prepare
def _values(gen, shape, dt):
    """Keys or values [..., heads, tokens, head_dim]: channels of a head differ in size."""
    channel = torch.exp(0.5 * torch.randn((shape[-3], 1, shape[-1]), generator=gen, device="cuda"))
    x = torch.empty(shape, dtype=dt, device="cuda")
    for i in range(0, shape[0], 4096):
        part = torch.randn((min(4096, shape[0] - i), *shape[1:]), generator=gen, device="cuda")
        x[i:i + 4096] = (part * channel).to(dt)
    return x


def _fill(s, K, V):
    """The cache of a state: pages 0 .. n - 1 hold what K and V [n, kv_heads, page, head_dim] are stored as."""
    c, n = s["case"], K.shape[0]
    if not own:
        s["pool"] = torch.empty((2, *K.shape), dtype=K.dtype, device="cuda")
        for plane, x in enumerate((K, V)):
            for i in range(0, n, 4096):
                s["pool"][plane, i:i + 4096] = _stored(x[i:i + 4096], c["bits"]).to(K.dtype)
        return
    from paper_2609_27373_gb300 import serve
    shape = dict(n_layers=1, n_pages=n, n_kv_heads=c["kv_heads"], page=c["page"], head_dim=c["head_dim"])
    whole = serve.PagedCache(n_slots=n, max_pages=1, dtype=K.dtype, bits=c["bits"], **shape)  # a sequence per page
    whole.table.copy_(torch.arange(n, dtype=torch.int32, device="cuda")[:, None])
    whole.lens.fill_(c["page"])
    whole.refs.fill_(1)
    whole.write(0, torch.arange(n, dtype=torch.int32, device="cuda"), None, K, V)
    s["cache"] = serve.PagedCache.over(whole.pool, s["table"], s["lens"], s["refs"], bits=c["bits"], page=c["page"],
                                       head_dim=c["head_dim"], dtype=K.dtype)


def _sequences(r, P, lens, shared, spans, spare=3):
    """table, lens, refs and slots of requests with the given lengths; those of span g (spans[g] .. spans[g + 1]) share
    their first shared[g] pages."""
    B = len(lens)
    need = sum(shared) + sum(-(-lens[i] // P) - shared[g] for g in range(len(shared)) for i in range(spans[g], spans[g + 1]))
    n_pages = need + spare
    ids = r.permutation(n_pages)
    slots = r.permutation(B + 2)[:B].astype(np.int32)
    table = np.zeros((B + 2, max(-(-x // P) for x in lens) + 1), np.int32)
    refs, length, n = np.zeros(n_pages, np.int32), np.zeros(B + 2, np.int32), 0
    for g in range(len(shared)):
        common, n = ids[n:n + shared[g]], n + shared[g]
        for i in range(spans[g], spans[g + 1]):
            k = -(-lens[i] // P) - shared[g]
            table[slots[i], :shared[g]] = common
            table[slots[i], shared[g]:shared[g] + k] = ids[n:n + k]
            n += k
            length[slots[i]] = lens[i]
    for slot in range(B + 2):
        np.add.at(refs, table[slot, :-(-length[slot] // P)], 1)
    return dict(table=torch.from_numpy(table).cuda(), lens=torch.from_numpy(length).cuda(),
                refs=torch.from_numpy(refs).cuda(), slots=torch.from_numpy(slots).cuda())


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _page_values(c, s, gen):
    """What the pages are filled with: keys and values [n_pages, kv_heads, page, head_dim]."""
    shape = (s["refs"].numel(), c["kv_heads"], c["page"], c["head_dim"])
    return _values(gen, shape, DTYPES[c["dtype"]]), _values(gen, shape, DTYPES[c["dtype"]])


# ------------------------------------------------- store: write, read back
def _store_sizes(c):
    """Tokens before, and new tokens, of each sequence."""
    B = c["batch"]
    before = [c["before"] - c["before"] * i // (2 * B) for i in range(B)]
    new = [max(1, c["q_len"] - c["q_len"] * (i % 4) // 5) for i in range(B)]
    return before, new


def _store_inputs(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    before, new = _store_sizes(c)
    order = r.permutation(c["batch"])
    before = [before[i] for i in order]
    lens = [a + b for a, b in zip(before, new)]
    s = dict(case=c, **_sequences(r, c["page"], lens, [0], [0, c["batch"]]))
    shape = (c["batch"], c["kv_heads"], c["q_len"], c["head_dim"])
    dt = DTYPES[c["dtype"]]
    s["K"], s["V"] = _values(gen, shape, dt), _values(gen, shape, dt)
    first = [max(0, n - KEPT) for n in before]
    s.update(new=_i32(new), first=_i32(first), count=_i32([n - f for n, f in zip(lens, first)]))
    rows = c["q_len"] + min(KEPT, c["before"])
    s["outK"] = torch.empty((c["batch"], c["kv_heads"], rows, c["head_dim"]), dtype=dt, device="cuda")
    s["outV"] = torch.empty_like(s["outK"])
    return s, _page_values(c, s, gen)


def _prepare_store(c, seed):
    s, pages = _store_inputs(c, seed)
    _fill(s, *pages)
    return s


def _run_store(s):
    if not own:
        _plain_write(s)
        return _plain_read(s)
    s["cache"].write(0, s["slots"], s["new"], s["K"], s["V"])
    s["cache"].read(0, s["outK"], s["outV"], s["slots"], s["first"], s["count"])
    return dict(K=s["outK"], V=s["outV"])


# ---------------------------------------------------------------- read
def _read_inputs(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B = c["batch"]
    lens = [max(1, c["length"] - c["length"] * i // (3 * B)) for i in range(B)]
    s = dict(case=c, **_sequences(r, c["page"], lens, [0], [0, B]))
    count = [max(1, min(lens[i], c["rows"] - c["rows"] * (i % 3) // 7)) for i in range(B)]
    first = [n - k if i % 2 == 0 else (n - k) // 3 for i, (n, k) in enumerate(zip(lens, count))]
    s.update(first=_i32(first), count=_i32(count))
    s["outK"] = torch.empty((B, c["kv_heads"], c["rows"], c["head_dim"]), dtype=DTYPES[c["dtype"]], device="cuda")
    s["outV"] = torch.empty_like(s["outK"])
    return s, _page_values(c, s, gen)


def _prepare_read(c, seed):
    s, pages = _read_inputs(c, seed)
    _fill(s, *pages)
    return s


def _run_read(s):
    if not own:
        return _plain_read(s)
    s["cache"].read(0, s["outK"], s["outV"], s["slots"], s["first"], s["count"])
    return dict(K=s["outK"], V=s["outV"])


# ---------------------------------------------------------------- attention
def _spans(c):
    """First request of each group, and one past the last (one group of everything when nothing is shared)."""
    g = max(1, c["groups"])
    return [c["batch"] * i // g for i in range(g + 1)]


def _prefix(c, g):
    """Tokens shared by group g: each further group's prompt is somewhat shorter."""
    return max(1, c["prefix"] - 37 * g) if c["groups"] else 0


def _lengths(c):
    """Tokens, and new tokens, of each request, in an order that the seed then shuffles within a group."""
    lens, new = [], []
    at = _spans(c)
    for g in range(len(at) - 1):
        n = at[g + 1] - at[g]
        for i in range(n):
            t = max(1, c["suffix"] * (i + 1) // n)
            lens.append((_prefix(c, g) if c["groups"] else c["prefix"] // 4) + t)
            new.append(min(t, 1 + i % c["q_len"]))
    return lens, new


def _plain_values(c):
    """Values that the plain form holds for the own part of the keys."""
    at, (lens, _) = _spans(c), _lengths(c)
    return sum((at[g + 1] - at[g]) * (max(lens[at[g]:at[g + 1]]) - _prefix(c, g) + c["page"])
               for g in range(len(at) - 1)) * c["kv_heads"] * c["head_dim"]


def _attend_inputs(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    P, at, B = c["page"], _spans(c), c["batch"]
    lens, new = _lengths(c)
    for g in range(len(at) - 1):
        o = at[g] + r.permutation(at[g + 1] - at[g])
        lens[at[g]:at[g + 1]], new[at[g]:at[g + 1]] = [lens[i] for i in o], [new[i] for i in o]
    s = dict(case=c, **_sequences(r, P, lens, [_prefix(c, g) // P for g in range(len(at) - 1)], at))
    # Logits of one or two units spread: a softmax that is neither flat nor one-hot.
    s["Q"] = torch.randn((B, c["heads"], c["q_len"], c["head_dim"]), generator=gen, device="cuda").to(DTYPES[c["dtype"]])
    s.update(O=torch.empty_like(s["Q"]), new=_i32(new), group_start=None, prefix_lens=None)
    if c["groups"]:
        s.update(group_start=_i32(at), prefix_lens=_i32([_prefix(c, g) for g in range(c["groups"])]))
    return s, _page_values(c, s, gen)


def _prepare_attend(c, seed):
    s, pages = _attend_inputs(c, seed)
    _fill(s, *pages)
    return s


def _plain_attend(s):
    c, P, D, KV, ql = s["case"], s["case"]["page"], s["case"]["head_dim"], s["case"]["kv_heads"], s["case"]["q_len"]
    R, at, O = c["heads"] // KV * ql, _spans(c), s["O"]
    own_max = c["suffix"] if c["groups"] else c["suffix"] + c["prefix"] // 4
    step = torch.arange(ql, device="cuda")
    for g in range(len(at) - 1):
        a, b = at[g], at[g + 1]
        n, np_ = b - a, _prefix(c, g) // P
        rows = s["slots"][a:b].long()
        new = s["new"][a:b, None]
        limit = torch.where(step < new, s["lens"][rows][:, None] - new + step + 1, 0)  # [n, ql] keys seen by a row
        limit = limit[:, None, :].expand(n, R // ql, ql).reshape(n, 1, R, 1)
        q = s["Q"][a:b].float().reshape(n, KV, R, D) * (1.0 / math.sqrt(D))
        last = -(-(_prefix(c, g) + own_max) // P)
        tab = s["table"][rows, np_:last].long()
        k, v = (x[tab].permute(0, 2, 1, 3, 4).reshape(n, KV, -1, D).float() for x in s["pool"])
        pos = np_ * P + torch.arange(k.shape[2], device="cuda")
        ss = torch.where(pos < limit, q @ k.transpose(2, 3), -math.inf)
        if np_:
            ids = s["table"][rows[0], :np_].long()
            kp, vp = (x[ids].permute(1, 0, 2, 3).reshape(KV, -1, D).float() for x in s["pool"])
            sp = (q.transpose(0, 1).reshape(KV, n * R, D) @ kp.transpose(1, 2)).reshape(KV, n, R, -1).transpose(0, 1)
            sp = torch.where(torch.arange(np_ * P, device="cuda") < limit, sp, -math.inf)
            m = torch.maximum(ss.amax(-1, True), sp.amax(-1, True))
        else:
            m = ss.amax(-1, True)
        m = torch.where(m == -math.inf, 0.0, m)
        e = torch.exp(ss - m)
        total, o = e.sum(-1, True), e @ v
        if np_:
            e = torch.exp(sp - m)
            total = total + e.sum(-1, True)
            o = o + (e.transpose(0, 1).reshape(KV, n * R, -1) @ vp).reshape(KV, n, R, D).transpose(0, 1)
        o = torch.where(total > 0, o / total, 0.0)
        O[a:b] = o.reshape(n, c["heads"], ql, D).to(O.dtype)
    return {"O": O}


def _run_attend(s):
    if not own:
        return _plain_attend(s)
    s["cache"].attend(0, s["Q"], s["O"], s["slots"], s["new"], s["group_start"], s["prefix_lens"])
    return {"O": s["O"]}


# ------------------------------------------------------------ in 64 bits
def _nearest(table, y):
    """The entries of an ascending table nearest to y >= 0 in size, ties to the even index."""
    t = torch.tensor(table, dtype=torch.float64, device=y.device)
    mid = (t[1:] + t[:-1]) / 2
    i = torch.searchsorted(mid, y)  # the number of midpoints below y
    tie = y == mid[torch.clamp(i, max=len(table) - 2)]
    return t[torch.where(tie & (i % 2 == 1), i + 1, i)]


def _floats(exponents, lowest, most):
    """0 and the numbers with 3 mantissa bits of the given number of binades, the lowest at 2^lowest, up to `most`."""
    out = [m * 2.0 ** (lowest - 3) for m in range(8)]
    for e in range(exponents):
        out += [(1 + m / 8) * 2.0 ** (lowest + e) for m in range(8)]
    return [x for x in out if x <= most]


def _exact_stored(x, bits):
    """What x is stored as, by looking every number up among all that there are; 32 bits hold it."""
    out = torch.empty(x.shape, dtype=torch.float32, device=x.device)
    for i in range(0, x.shape[0], 512):
        g = x[i:i + 512].double().reshape(*x[i:i + 512].shape[:-1], -1, 16)
        a = g.abs().amax(-1, True).contiguous()
        if bits == 4:
            s = _nearest(_floats(28, -14, 10240.0), a / torch.full_like(a, 6.0))
            y = torch.where(s > 0, g.abs() / torch.where(s > 0, s, 1.0), 0.0)
            q = _nearest([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], y)
        else:
            powers = torch.tensor([2.0 ** k for k in range(-15, 8)], dtype=torch.float64, device=x.device)
            s = powers[torch.clamp(torch.searchsorted(448 * powers, a), max=22)]
            q = _nearest(_floats(15, -6, 448.0), g.abs() / s)
        out[i:i + 512] = (torch.sign(g) * q * s).reshape(x[i:i + 512].shape).float()
    return out


def _exact_sequence(s, pages, slot, n):
    """Keys and values [n, kv_heads, head_dim] of the first n tokens of a sequence."""
    P = s["case"]["page"]
    at = torch.arange(n, device="cuda")
    page, off = s["table"][slot].long()[at // P], at % P
    return [x[page, :, off] for x in pages]


def _exact_rows(s, pages):
    """The rows first .. first + count of each sequence."""
    out = [torch.zeros(s["outK"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    lens = s["lens"].tolist()
    for b, (slot, f, n) in enumerate(zip(s["slots"].tolist(), s["first"].tolist(), s["count"].tolist())):
        for o, x in zip(out, _exact_sequence(s, pages, slot, lens[slot])):
            o[b, :, :n] = x[f:f + n].double().transpose(0, 1)
    return dict(K=out[0], V=out[1])


def _exact_store(c, seed):
    s, pages = _store_inputs(c, seed)
    pages = [_exact_stored(x, c["bits"]) for x in pages]
    lens = s["lens"].tolist()
    for b, (slot, n) in enumerate(zip(s["slots"].tolist(), s["new"].tolist())):
        at = torch.arange(lens[slot] - n, lens[slot], device="cuda")
        page, off = s["table"][slot].long()[at // c["page"]], at % c["page"]
        for x, new in zip(pages, (s["K"], s["V"])):
            x[page, :, off] = _exact_stored(new[b, :, :n].transpose(0, 1), c["bits"])
    return _exact_rows(s, pages)


def _exact_read(c, seed):
    s, pages = _read_inputs(c, seed)
    return _exact_rows(s, [_exact_stored(x, c["bits"]) for x in pages])


def _exact_attend(c, seed):
    s, pages = _attend_inputs(c, seed)
    pages = [_exact_stored(x, c["bits"]) for x in pages]
    D, KV = c["head_dim"], c["kv_heads"]
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lens, new = s["lens"].tolist(), s["new"].tolist()
    for i, slot in enumerate(s["slots"].tolist()):
        n = lens[slot]
        k, v = (x.double() for x in _exact_sequence(s, pages, slot, n))
        for t in range(new[i]):
            seen = n - new[i] + t + 1
            q = s["Q"][i, :, t].double().reshape(KV, -1, D)
            w = torch.softmax(torch.einsum("kgd,nkd->kgn", q, k[:seen]) / math.sqrt(D), dim=-1)
            O[i, :, t] = torch.einsum("kgn,nkd->kgd", w, v[:seen]).reshape(-1, D)
    return {"O": O}


# --------------------------------------------------------------- the module
def prepare(case, seed):
    return dict(attend=_prepare_attend, store=_prepare_store, read=_prepare_read)[case["kind"]](case, seed)


def run(state):
    return dict(attend=_run_attend, store=_run_store, read=_run_read)[state["case"]["kind"]](state)


def exact(case, seed):
    return dict(attend=_exact_attend, store=_exact_store, read=_exact_read)[case["kind"]](case, seed)


def work(case):
    c = case
    packed = c["kv_heads"] * c["head_dim"] * (2 * c["bits"] + 1) // 8  # bytes of a token's keys, and of its values
    if c["kind"] == "attend":
        at, (lens, new) = _spans(c), _lengths(c)
        keys = 0
        for g in range(len(at) - 1):
            shared = _prefix(c, g) // c["page"] * c["page"]
            keys += shared + sum(lens[i] - shared for i in range(at[g], at[g + 1]))
        seen = sum(t * n - t * (t - 1) // 2 for t, n in zip(new, lens))
        return dict(bytes=2 * packed * keys + 2 * c["heads"] * c["head_dim"] * (sum(new) + c["batch"] * c["q_len"]),
                    flops=4 * c["heads"] * c["head_dim"] * seen)
    values = 2 * c["kv_heads"] * c["head_dim"]  # of a token
    if c["kind"] == "store":
        before, new = _store_sizes(c)
        rows = c["batch"] * (c["q_len"] + min(KEPT, c["before"]))
        back = sum(n + min(KEPT, b) for n, b in zip(new, before))
        # New rows are read and stored, then read again with a few older ones and written as values.
        return dict(bytes=sum(new) * (2 * values + 2 * packed) + back * 2 * packed + rows * 2 * values,
                    flops=4 * values * sum(new) + values * back)
    count = sum(max(1, c["rows"] - c["rows"] * (i % 3) // 7) for i in range(c["batch"]))
    return dict(bytes=count * 2 * packed + c["batch"] * c["rows"] * 2 * values, flops=values * count)
