"""Workloads of the serving operators: attention of a batch over a paged cache with shared prefixes, the cache's own
operations (fork, extend, write, drop, compact), and the verification of drafted tokens.

Each workload can run in its plain form (elementary torch operations in 32 bits) or through the package; `own`
chooses.  Sizes are those of this package's configurations (4 heads of 64; 32 heads of 128 at 4K; 55 heads of 96;
32 query heads over 8 key heads of 128 at 32K) with generic batches, page sizes and vocabularies.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # One prompt sampled twice: a handful of cached tokens, where only latency counts.
        dict(name="attend_small", kind="attend", dtype="bf16", heads=4, kv_heads=4, head_dim=64, page=16, groups=1,
             batch=2, prefix=512, suffix=40, q_len=1),
        # 16 continuations of one 4K prompt, one token each, every query head with its own keys.
        dict(name="attend_4k", kind="attend", dtype="bf16", heads=32, kv_heads=32, head_dim=128, page=64, groups=1,
             batch=16, prefix=4096, suffix=300, q_len=1),
        # Ragged drafts of up to 3 tokens, 55 heads of 96, a prefix that ends inside a page, fp16.
        dict(name="attend_odd_d96", kind="attend", dtype="fp16", heads=55, kv_heads=55, head_dim=96, page=32, groups=1,
             batch=7, prefix=4001, suffix=777, q_len=3),
        # A long document asked 64 questions: 32K shared tokens, grouped heads, one token a request.
        dict(name="attend_32k_gqa", kind="attend", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=64, groups=1,
             batch=64, prefix=32768, suffix=1024, q_len=1),
        # Two system prompts, 48 requests that verify up to 4 drafted tokens each.
        dict(name="attend_drafts", kind="attend", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=128, groups=2,
             batch=48, prefix=16384, suffix=2000, q_len=5),
        # Many short samples of one prompt: 1024 query rows a key head, bound by the products.
        dict(name="attend_rollouts", kind="attend", dtype="bf16", heads=32, kv_heads=8, head_dim=128, page=64, groups=1,
             batch=256, prefix=8192, suffix=128, q_len=1),
        # A few children of one sequence in a small cache.
        dict(name="branch_small", kind="branch", dtype="bf16", layers=1, kv_heads=4, head_dim=64, page=16, families=1,
             children=3, prefix=500, q_len=2),
        # Four prompts with 31 children each, every sequence grown by a ragged draft, eight layers.
        dict(name="branch_wide", kind="branch", dtype="bf16", layers=8, kv_heads=8, head_dim=128, page=64, families=4,
             children=31, prefix=8100, q_len=5),
        # Two of a few short requests end and their pages are closed up.
        dict(name="compact_small", kind="compact", dtype="bf16", layers=1, kv_heads=4, head_dim=64, page=16, slots=5,
             length=300, spare=0.2),
        # Half of the requests of a large cache end; the rest moves to its front.
        dict(name="compact_large", kind="compact", dtype="bf16", layers=8, kv_heads=8, head_dim=128, page=16, slots=96,
             length=1500, spare=0.2),
        # One request with four drafted tokens and a small vocabulary.
        dict(name="verify_small", kind="verify", dtype="bf16", batch=1, k=4, vocab=32000),
        # A full batch with an odd, large vocabulary in 32 bits.
        dict(name="verify_large", kind="verify", dtype="fp32", batch=160, k=6, vocab=131075),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attend", "attend", "attend", "branch", "compact", "verify"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    heads, kv_heads, head_dim = rng.choice([(4, 4, 64), (32, 32, 128), (55, 55, 96), (32, 8, 128), (8, 2, 64), (24, 4, 96)])
    page = rng.choice([16, 32, 64, 128])
    if kind == "attend":
        c = dict(kind=kind, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page,
                 groups=rng.choice([0, 1, 1, 1, 2, 3]), batch=log(1, 256), prefix=log(1, 32768), suffix=log(1, 2048),
                 q_len=rng.choice([1, 1, 2, 3, 4, 5, 8]))
        c["groups"] = min(c["groups"], c["batch"])
        c["suffix"] = max(c["suffix"], c["q_len"])
        while work(c)["flops"] > 3e10 or work(c)["bytes"] > 6e8 or _plain_values(c) > 4e8:
            c["batch"], c["prefix"] = max(c["groups"], 1, c["batch"] * 2 // 3), max(1, c["prefix"] * 3 // 4)
        return c
    if kind == "branch":
        c = dict(kind=kind, dtype=dtype, layers=rng.randint(1, 8), kv_heads=kv_heads, head_dim=head_dim, page=page,
                 families=rng.randint(1, 4), children=log(1, 31), prefix=log(1, 8192), q_len=rng.randint(1, 8))
        while work(c)["bytes"] > 2.4e8:
            c["children"] = max(1, c["children"] // 2)
            c["layers"] = max(1, c["layers"] - 1)
        return c
    if kind == "compact":
        c = dict(kind=kind, dtype=dtype, layers=rng.randint(1, 8), kv_heads=kv_heads, head_dim=head_dim, page=page,
                 slots=log(3, 96), length=log(20, 1500), spare=round(rng.uniform(0.05, 0.6), 2))
        while work(c)["bytes"] > 1e9:
            c["length"] = c["length"] * 2 // 3
            c["layers"] = max(1, c["layers"] - 1)
        return c
    return dict(kind=kind, dtype=rng.choice(["bf16", "fp16", "fp32"]), batch=log(1, 160), k=rng.randint(1, 6),
                vocab=log(1000, 131072))


# ---------------------------------------------------------------- attention
def _spans(c):
    """First request of each group, and one past the last (one group of everything when nothing is shared)."""
    g = max(1, c["groups"])
    return [c["batch"] * i // g for i in range(g + 1)]


def _prefix(c, g):
    """Tokens shared by group g: each further group's prompt is somewhat shorter."""
    return max(1, c["prefix"] - 37 * g) if c["groups"] else 0


def _own_tokens(c):
    """Own tokens and new tokens of each request, in an order that the seed then shuffles within a group."""
    own_t, new_t = [], []
    at = _spans(c)
    for g in range(len(at) - 1):
        n = at[g + 1] - at[g]
        for i in range(n):
            t = max(1, c["suffix"] * (i + 1) // n)
            own_t.append(t)
            new_t.append(min(t, 1 + i % c["q_len"]))
    return own_t, new_t


def _lengths(c):
    own_t, new_t = _own_tokens(c)
    at, base = _spans(c), []
    for g in range(len(at) - 1):
        base += [_prefix(c, g) if c["groups"] else c["prefix"] // 4] * (at[g + 1] - at[g])
    return [b + t for b, t in zip(base, own_t)], new_t


def _plain_values(c):
    """Values that the plain form holds for the own part of the keys."""
    at, (lens, _) = _spans(c), _lengths(c)
    return sum((at[g + 1] - at[g]) * (max(lens[at[g]:at[g + 1]]) - _prefix(c, g) + c["page"])
               for g in range(len(at) - 1)) * c["kv_heads"] * c["head_dim"]


def _prepare_attend(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    P, at, B = c["page"], _spans(c), c["batch"]
    lens, new = _lengths(c)
    for g in range(len(at) - 1):
        o = at[g] + r.permutation(at[g + 1] - at[g])
        lens[at[g]:at[g + 1]], new[at[g]:at[g + 1]] = [lens[i] for i in o], [new[i] for i in o]
    shared = [_prefix(c, g) // P for g in range(len(at) - 1)]
    need = sum(shared) + sum(-(-lens[i] // P) - shared[g] for g in range(len(shared)) for i in range(at[g], at[g + 1]))
    n_pages = need + 3
    ids = r.permutation(n_pages)
    max_pages = max(-(-x // P) for x in lens) + 1
    n_slots = B + 2
    slots = r.permutation(n_slots)[:B].astype(np.int32)
    table, refs, n = np.zeros((n_slots, max_pages), np.int32), np.zeros(n_pages, np.int32), 0
    length = np.zeros(n_slots, np.int32)
    for g in range(len(shared)):
        common, n = ids[n:n + shared[g]], n + shared[g]
        for i in range(at[g], at[g + 1]):
            k = -(-lens[i] // P) - shared[g]
            table[slots[i], :shared[g]] = common
            table[slots[i], shared[g]:shared[g] + k] = ids[n:n + k]
            n += k
            length[slots[i]] = lens[i]
    for s in range(n_slots):
        np.add.at(refs, table[s, :-(-length[s] // P)], 1)
    dt = DTYPES[c["dtype"]]
    # Logits of unit spread a step: a softmax that is neither flat nor one-hot.
    pool = torch.randn((2, n_pages, c["kv_heads"], P, c["head_dim"]), generator=gen, device="cuda", dtype=dt)
    Q = torch.randn((B, c["heads"], c["q_len"], c["head_dim"]), generator=gen, device="cuda", dtype=dt) * 1.5
    s = dict(case=c, pool=pool, Q=Q, O=torch.empty_like(Q),
             table=torch.from_numpy(table).cuda(), lens=torch.from_numpy(length).cuda(),
             refs=torch.from_numpy(refs).cuda(), slots=torch.from_numpy(slots).cuda(),
             new=torch.tensor(new, dtype=torch.int32, device="cuda"), group_start=None, prefix_lens=None)
    if c["groups"]:
        s["group_start"] = torch.tensor(at, dtype=torch.int32, device="cuda")
        s["prefix_lens"] = torch.tensor([_prefix(c, g) for g in range(c["groups"])], dtype=torch.int32, device="cuda")
    if own:
        from paper_2609_27373_gb300 import serve
        s["cache"] = serve.PagedCache.over(pool, s["table"], s["lens"], s["refs"])
    return s


def _plain_attend(s):
    c, P, D, KV, ql = s["case"], s["case"]["page"], s["case"]["head_dim"], s["case"]["kv_heads"], s["case"]["q_len"]
    R, at, O = c["heads"] // KV * ql, _spans(c), s["O"]
    own_max = [c["suffix"] if c["groups"] else c["suffix"] + c["prefix"] // 4] * (len(at) - 1)
    step = torch.arange(ql, device="cuda")
    for g in range(len(at) - 1):
        a, b = at[g], at[g + 1]
        n, np_ = b - a, _prefix(c, g) // P
        rows = s["slots"][a:b].long()
        new = s["new"][a:b, None]
        limit = torch.where(step < new, s["lens"][rows][:, None] - new + step + 1, 0)  # [n, ql] keys seen by a row
        limit = limit[:, None, :].expand(n, R // ql, ql).reshape(n, 1, R, 1)
        q = s["Q"][a:b].float().reshape(n, KV, R, D) * (1.0 / math.sqrt(D))
        last = -(-(_prefix(c, g) + own_max[g]) // P)
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


def _exact_attend(c, seed):
    s = _prepare_attend(c, seed)
    D, KV = c["head_dim"], c["kv_heads"]
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lens, slots, new = s["lens"].tolist(), s["slots"].tolist(), s["new"].tolist()
    for i, slot in enumerate(slots):
        n = lens[slot]
        where = torch.arange(n, device="cuda")
        page, off = s["table"][slot].long()[where // c["page"]], where % c["page"]
        k, v = s["pool"][0, page, :, off].double(), s["pool"][1, page, :, off].double()  # [n, KV, D]
        for t in range(new[i]):
            seen = n - new[i] + t + 1
            q = s["Q"][i, :, t].double().reshape(KV, -1, D)
            w = torch.softmax(torch.einsum("kgd,nkd->kgn", q, k[:seen]) / math.sqrt(D), dim=-1)
            O[i, :, t] = torch.einsum("kgn,nkd->kgd", w, v[:seen]).reshape(-1, D)
    return {"O": O}


# ------------------------------------------------- fork, extend and write
def _branch_sizes(c):
    """Sequences, their tokens before and the tokens each is grown by."""
    F, C = c["families"], c["children"]
    before = [max(1, c["prefix"] - 29 * f) for f in range(F)]
    length = before + [before[f] for f in range(F) for _ in range(C)]
    grow = [i % (c["q_len"] + 1) for i in range(F * (C + 1))]
    grow[0] = c["q_len"]
    return before, length, grow


def _prepare_branch(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    P, F, C = c["page"], c["families"], c["children"]
    before, length, grow = _branch_sizes(c)
    B = len(length)
    n_slots = B + 3
    order = r.permutation(n_slots)[:B].astype(np.int32)
    max_pages = -(-(max(length) + c["q_len"]) // P) + 1
    used = sum(-(-x // P) for x in before)
    n_pages = used + B * (2 + c["q_len"] // P) + 7
    ids = r.permutation(n_pages)[:used]
    table, lens, refs, n = np.zeros((n_slots, max_pages), np.int32), np.zeros(n_slots, np.int32), np.zeros(n_pages, np.int32), 0
    for f in range(F):
        k = -(-before[f] // P)
        table[order[f], :k], lens[order[f]] = ids[n:n + k], before[f]
        refs[ids[n:n + k]] = 1
        n += k
    meta = torch.from_numpy(np.concatenate([table.reshape(-1), lens, refs])).cuda()
    dt = DTYPES[c["dtype"]]
    shape = (c["layers"], B, c["kv_heads"], c["q_len"], c["head_dim"])
    s = dict(case=c, pool=torch.randn((2 * c["layers"], n_pages, c["kv_heads"], P, c["head_dim"]), generator=gen, device="cuda", dtype=dt),
             K=torch.randn(shape, generator=gen, device="cuda", dtype=dt), V=torch.randn(shape, generator=gen, device="cuda", dtype=dt),
             src=torch.from_numpy(np.repeat(order[:F], C)).cuda(), dst=torch.from_numpy(order[F:]).cuda(),
             slots=torch.from_numpy(order).cuda(), grow=torch.from_numpy(r.permutation(np.array(grow, np.int32))).cuda())
    _with_meta(s, meta, n_slots, max_pages, n_pages)
    return s


def _with_meta(s, meta, n_slots, max_pages, n_pages):
    """The cache's bookkeeping as views of one buffer, which a pass sets back to where it was first."""
    s["meta0"], s["meta"] = meta, meta.clone()
    s["table"] = s["meta"][:n_slots * max_pages].view(n_slots, max_pages)
    s["lens"] = s["meta"][n_slots * max_pages:][:n_slots]
    s["refs"] = s["meta"][n_slots * (max_pages + 1):]
    if own:
        from paper_2609_27373_gb300 import serve
        s["cache"] = serve.PagedCache.over(s["pool"], s["table"], s["lens"], s["refs"])


def _count_refs(refs, table, used, by):
    """refs += by for the first `used` entries of each row of a table."""
    held = torch.arange(table.shape[1], device="cuda") < used[:, None]
    refs.scatter_add_(0, torch.where(held, table, 0).reshape(-1).long(), held.reshape(-1).int() * by)


def _run_branch(s):
    c, P = s["case"], s["case"]["page"]
    s["meta"].copy_(s["meta0"])
    if own:
        cache = s["cache"]
        cache.fork(s["src"], s["dst"])
        granted = cache.extend(s["slots"], s["grow"])
        for layer in range(c["layers"]):
            cache.write(layer, s["slots"], granted, s["K"][layer], s["V"][layer])
        return dict(table=s["table"], lens=s["lens"], refs=s["refs"], granted=granted, pool=s["pool"])
    table, lens, refs, pool = s["table"], s["lens"], s["refs"], s["pool"]
    # fork: the child's row is its parent's, and every page has one more holder
    src, dst = s["src"].long(), s["dst"].long()
    table[dst], lens[dst] = table[src], lens[src]
    _count_refs(refs, table[dst], (lens[dst] + P - 1) // P, 1)
    # extend: new pages from the lowest free ones; a shared page that is not full is copied for whom it grows
    slots, grow = s["slots"].long(), s["grow"]
    old = lens[slots]
    tail = torch.where(old % P > 0, table[slots, old // P], 0)
    copy = (grow > 0) & (old % P > 0) & (refs[tail.long()] > 1)
    need = (old + grow + P - 1) // P - (old + P - 1) // P + copy.int()
    upto = torch.cumsum(need, 0)
    free = torch.nonzero(refs == 0)[:, 0]
    granted = torch.where((need == 0) | (upto <= free.numel()), grow, 0)
    first = torch.where(copy, old // P, (old + P - 1) // P)
    k = torch.arange(2 + c["q_len"] // P, device="cuda")
    new = torch.nonzero((k < need[:, None]) & (granted > 0)[:, None])
    page = free[(upto - need)[new[:, 0]] + new[:, 1]]
    moved = torch.nonzero(copy & (granted > 0))[:, 0]
    a, b, rows = tail[moved].long(), free[(upto - need)[moved]], (old % P)[moved]
    inside = torch.arange(P, device="cuda") < rows[:, None]
    pool[:, b] = torch.where(inside[None, :, None, :, None], pool[:, a], pool[:, b])
    refs.scatter_add_(0, a, torch.full_like(a, -1, dtype=torch.int32))
    table[slots[new[:, 0]], first[new[:, 0]].long() + new[:, 1]] = page.int()
    refs[page] = 1
    lens[slots] = old + granted
    # write: the new tokens' keys and values, layer by layer
    at = torch.nonzero(torch.arange(c["q_len"], device="cuda") < granted[:, None])
    pos = old[at[:, 0]] + at[:, 1]
    to = table[slots[at[:, 0]], (pos // P).long()].long()
    for layer in range(c["layers"]):
        pool[2 * layer, to, :, (pos % P).long()] = s["K"][layer][at[:, 0], :, at[:, 1]]
        pool[2 * layer + 1, to, :, (pos % P).long()] = s["V"][layer][at[:, 0], :, at[:, 1]]
    return dict(table=table, lens=lens, refs=refs, granted=granted, pool=pool)


def _exact_branch(c, seed):
    """One sequence after another, on lists."""
    s = _prepare_branch(c, seed)
    P, table, lens, refs = c["page"], s["table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        table[b], lens[b] = list(table[a]), lens[a]
        for j in range(-(-lens[b] // P)):
            refs[table[b][j]] += 1
    free, held, given = [i for i, x in enumerate(refs) if x == 0], list(refs), []
    for slot, n in zip(s["slots"].tolist(), s["grow"].tolist()):
        have, want = -(-lens[slot] // P), -(-(lens[slot] + n) // P)
        if n and lens[slot] % P and held[table[slot][have - 1]] > 1:
            refs[table[slot][have - 1]] -= 1
            have -= 1
        for j in range(have, want):
            table[slot][j] = free.pop(0)
            refs[table[slot][j]] = 1
        lens[slot] += n
        given.append(n)
    return dict(table=np.array(table, np.int32), lens=np.array(lens, np.int32), refs=np.array(refs, np.int32),
                granted=np.array(given, np.int32), pool=None)


# -------------------------------------------------------- drop and compact
def _compact_sizes(c):
    """Tokens of each sequence, and how many of them go: half end, a quarter is cut short."""
    length = [max(1, c["length"] * (i + 2) // (c["slots"] + 1)) for i in range(c["slots"])]
    gone = [length[i] if i % 4 < 2 else min(length[i], 1 + c["length"] // 7) if i % 4 == 2 else 0 for i in range(c["slots"])]
    return length, gone


def _compact_pages(c):
    P, (length, gone) = c["page"], _compact_sizes(c)
    used = sum(-(-x // P) for x in length)
    left = sum(-(-(x - y) // P) for x, y in zip(length, gone))
    return used, left, int(used * (1 + c["spare"])) + 2


def _prepare_compact(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    P, (length, gone), (used, _, n_pages) = c["page"], _compact_sizes(c), _compact_pages(c)
    n_slots = c["slots"] + 2
    order = r.permutation(n_slots)[:c["slots"]].astype(np.int32)
    ids, n = r.permutation(n_pages)[:used], 0
    table, lens, refs = np.zeros((n_slots, max(-(-x // P) for x in length) + 1), np.int32), np.zeros(n_slots, np.int32), np.zeros(n_pages, np.int32)
    for i, slot in enumerate(order):
        k = -(-length[i] // P)
        table[slot, :k], lens[slot] = ids[n:n + k], length[i]
        n += k
    refs[ids] = 1
    pool = torch.randn((2 * c["layers"], n_pages, c["kv_heads"], P, c["head_dim"]), generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
    s = dict(case=c, pool=pool, slots=torch.from_numpy(order).cuda(), gone=torch.tensor(gone, dtype=torch.int32, device="cuda"))
    _with_meta(s, torch.from_numpy(np.concatenate([table.reshape(-1), lens, refs])).cuda(), n_slots, table.shape[1], n_pages)
    return s


def _run_compact(s):
    s["meta"].copy_(s["meta0"])
    if own:
        s["cache"].drop(s["slots"], s["gone"])
        remap, n_live = s["cache"].compact()
        return dict(table=s["table"], lens=s["lens"], refs=s["refs"], remap=remap, n_live=n_live, pool=s["pool"])
    P, table, lens, refs, pool = s["case"]["page"], s["table"], s["lens"], s["refs"], s["pool"]
    # drop: the pages past a sequence's new end lose a holder
    slots = s["slots"].long()
    old = lens[slots]
    new = torch.clamp(old - s["gone"], min=0)
    _count_refs(refs, table[slots], (old + P - 1) // P, -1)
    _count_refs(refs, table[slots], (new + P - 1) // P, 1)
    lens[slots] = new
    # compact: the k-th page in use past the first n_live goes to the k-th hole among them
    live = refs > 0
    n_live = live.sum().int().reshape(1)
    place = torch.arange(refs.numel(), device="cuda")
    src, dst = torch.nonzero(live & (place >= n_live))[:, 0], torch.nonzero(~live & (place < n_live))[:, 0]
    pool[:, dst] = pool[:, src]
    remap = torch.where(live, place, -1).int()
    remap[src] = dst.int()
    refs[dst] = refs[src]
    refs[src] = 0
    held = torch.arange(table.shape[1], device="cuda") < ((lens + P - 1) // P)[:, None]
    table.copy_(torch.where(held, remap[table.long()], table))
    return dict(table=table, lens=lens, refs=refs, remap=remap, n_live=n_live, pool=pool)


def _exact_compact(c, seed):
    s = _prepare_compact(c, seed)
    P, table, lens, refs = c["page"], s["table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    for slot, n in zip(s["slots"].tolist(), s["gone"].tolist()):
        keep = max(0, lens[slot] - n)
        for j in range(-(-keep // P), -(-lens[slot] // P)):
            refs[table[slot][j]] -= 1
        lens[slot] = keep
    n_live = sum(x > 0 for x in refs)
    to = {i: i for i, x in enumerate(refs) if x > 0}
    holes = [i for i in range(n_live) if refs[i] == 0]
    for i in range(n_live, len(refs)):
        if refs[i] > 0:
            to[i] = holes.pop(0)
            refs[to[i]], refs[i] = refs[i], 0
    for slot in range(len(lens)):
        for j in range(-(-lens[slot] // P)):
            table[slot][j] = to[table[slot][j]]
    remap = [to.get(i, -1) for i in range(len(refs))]
    return dict(table=np.array(table, np.int32), lens=np.array(lens, np.int32), refs=np.array(refs, np.int32),
                remap=np.array(remap, np.int32), n_live=np.array([n_live], np.int32), pool=None)


# ------------------------------------------------------------ verification
def _prepare_verify(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, K, V, dt = c["batch"], c["k"], c["vocab"], DTYPES[c["dtype"]]
    logits = torch.randn((B, K + 1, V), generator=gen, device="cuda") * 2.5
    p = torch.softmax(logits, -1)
    # The draft model is near the target, so that most drafted tokens stand.
    q = torch.softmax(logits[:, :K] + 0.4 * torch.randn((B, K, V), generator=gen, device="cuda"), -1)
    draft = torch.multinomial(q.reshape(B * K, V), 1, generator=gen).reshape(B, K).int()
    n_draft = torch.tensor([K if i % 3 < 2 else i % (K + 1) for i in range(B)], dtype=torch.int32, device="cuda")
    return dict(case=c, p=p.to(dt), q=q.to(dt), draft=draft, n_draft=n_draft,
                u_accept=torch.rand((B, K), generator=gen, device="cuda"),
                u_sample=torch.rand((B,), generator=gen, device="cuda"))


def _run_verify(s):
    if own:
        from paper_2609_27373_gb300 import serve
        accepted, tokens = serve.verify_draft(s["p"], s["q"], s["draft"], s["n_draft"], s["u_accept"], s["u_sample"])
        return dict(accepted=accepted, tokens=tokens)
    p, q, draft, n_draft = s["p"], s["q"], s["draft"].long(), s["n_draft"].long()
    B, K, V = q.shape
    step = torch.arange(K + 1, device="cuda")
    px = p[:, :K].gather(2, draft[..., None])[..., 0].float()
    qx = q.gather(2, draft[..., None])[..., 0].float()
    stands = (s["u_accept"] * qx < px) & (step[:K] < n_draft[:, None])
    acc = torch.cumprod(stands.int(), 1).sum(1)
    row = torch.arange(B, device="cuda")
    pr = p[row, acc].float()
    qr = q[row, torch.clamp(acc, max=K - 1)].float()
    left = torch.where((acc < n_draft)[:, None], torch.clamp(pr - qr, min=0.0), pr)

    def weights(x):  # fixed point, so that sums do not depend on their order
        return (torch.clamp(x, 0.0, 1.0) * 2.0 ** 40).long()

    w = weights(left)
    w = torch.where(w.sum(1, True) > 0, w, weights(pr))
    total = w.sum(1)
    u = (torch.clamp(s["u_sample"], 0.0, 1.0 - 2.0 ** -24) * 2.0 ** 24).long()
    at = (total >> 24) * u + (((total & 0xFFFFFF) * u) >> 24)
    token = (torch.cumsum(w, 1) <= at[:, None]).sum(1)
    token = torch.where(total > 0, token, -1)
    tokens = torch.where(step < acc[:, None], torch.nn.functional.pad(draft, (0, 1)), torch.where(step == acc[:, None], token[:, None], -1))
    return dict(accepted=acc.int(), tokens=tokens.int())


def _exact_verify(c, seed):
    s = _prepare_verify(c, seed)
    draft, n_draft, ua, us = s["draft"].tolist(), s["n_draft"].tolist(), s["u_accept"].cpu().numpy(), s["u_sample"].tolist()
    accepted, tokens = [], []
    for b in range(c["batch"]):
        n, said = 0, []
        while n < n_draft[b]:
            x = draft[b][n]
            if not ua[b, n] * np.float32(s["q"][b, n, x].item()) < np.float32(s["p"][b, n, x].item()):
                break
            said.append(x)
            n += 1
        p = s["p"][b, n].double().cpu().numpy()
        r = p if n == n_draft[b] else np.maximum(p.astype(np.float32) - s["q"][b, n].float().cpu().numpy(), 0).astype(np.float64)
        w = np.floor(np.minimum(r, 1.0) * 2.0 ** 40).astype(np.int64)
        if not w.any():
            w = np.floor(np.minimum(p, 1.0) * 2.0 ** 40).astype(np.int64)
        cum = np.cumsum(w)
        at = (int(cum[-1]) * int(us[b] * 2 ** 24)) >> 24
        accepted.append(n)
        tokens.append(said + [int(np.searchsorted(cum, at, side="right")) if cum[-1] else -1] + [-1] * (c["k"] - n))
    return dict(accepted=np.array(accepted, np.int32), tokens=np.array(tokens, np.int32))


# --------------------------------------------------------------- the module
def prepare(case, seed):
    return dict(attend=_prepare_attend, branch=_prepare_branch, compact=_prepare_compact, verify=_prepare_verify)[case["kind"]](case, seed)


def run(state):
    return dict(attend=_run_attend, branch=_run_branch, compact=_run_compact, verify=_run_verify)[state["case"]["kind"]](state)


def exact(case, seed):
    return dict(attend=_exact_attend, branch=_exact_branch, compact=_exact_compact, verify=_exact_verify)[case["kind"]](case, seed)


def work(case):
    c = case
    if c["kind"] == "attend":
        at, (lens, new) = _spans(c), _lengths(c)
        keys = 0
        for g in range(len(at) - 1):
            shared = _prefix(c, g) // c["page"] * c["page"]
            keys += shared + sum(lens[i] - shared for i in range(at[g], at[g + 1]))
        seen = sum(t * n - t * (t - 1) // 2 for t, n in zip(new, lens))
        return dict(bytes=4 * c["kv_heads"] * c["head_dim"] * keys + 2 * c["heads"] * c["head_dim"] * (sum(new) + c["batch"] * c["q_len"]),
                    flops=4 * c["heads"] * c["head_dim"] * seen)
    if c["kind"] == "verify":
        size = 4 if c["dtype"] == "fp32" else 2
        # Two rows where a draft is turned down, one where all of it stands (about one in three here).
        return dict(bytes=int(c["batch"] * c["vocab"] * size * 1.67) + c["batch"] * (2 * size * c["k"] + 4 * (3 * c["k"] + 4)),
                    flops=3 * c["batch"] * c["vocab"])
    P = c["page"]
    token = 4 * c["layers"] * c["kv_heads"] * c["head_dim"]
    if c["kind"] == "branch":
        before, length, grow = _branch_sizes(c)
        # Rows of shared last pages are copied for about all that grow; new rows are read and written.
        copied = sum(n % P for n in length) * c["q_len"] / (c["q_len"] + 1)
        entries = sum(-(-n // P) for n in length[len(before):])
        return dict(bytes=int(2 * token * (copied + sum(grow)) + 16 * entries + 16 * len(length)), flops=0)
    used, left, n_pages = _compact_pages(c)
    moves = left * (1 - left / n_pages)
    return dict(bytes=int(2 * token * P * moves + 8 * n_pages + 12 * used), flops=0)
