"""Plain models of the serving operators: a paged cache as Python lists, its
attention in fp64, and the verification rule in Python integers."""
import math

import numpy as np
import torch


class ListCache:
    """The cache's rules, one entry after another (a faulty entry is passed over and counted)."""

    def __init__(self, n_pages, page, n_slots, max_pages):
        self.page, self.max_pages, self.faults, self.starved = page, max_pages, 0, 0
        self.rows = [[] for _ in range(n_slots)]
        self.lens = [0] * n_slots
        self.refs = [0] * n_pages

    def pages(self, n):
        return -(-n // self.page)

    def fork(self, src, dst):
        for i, (s, d) in enumerate(zip(src, dst)):
            if s < 0 or d < 0:
                continue
            if s >= len(self.lens) or d >= len(self.lens) or dst.count(d) > 1 or d in src:
                self.faults += 1
                continue
            for g in self.rows[d]:
                self.refs[g] -= 1
            self.rows[d], self.lens[d] = list(self.rows[s]), self.lens[s]
            for g in self.rows[d]:
                self.refs[g] += 1

    def extend(self, slots, n_new):
        """Returns granted, and the copies (from page, to page, rows)."""
        granted, copies, spent = [], [], 0
        free = [g for g, r in enumerate(self.refs) if r == 0]
        held = list(self.refs)
        for s, n in zip(slots, n_new):
            give = 0
            if s >= 0:
                if s >= len(self.lens) or slots.count(s) > 1 or n < 0:
                    self.faults += 1
                elif self.lens[s] + n > self.max_pages * self.page:
                    self.starved += 1
                else:
                    rest = self.lens[s] % self.page
                    copy = n > 0 and rest > 0 and held[self.rows[s][-1]] > 1
                    need = self.pages(self.lens[s] + n) - self.pages(self.lens[s]) + copy
                    spent += need
                    if need == 0 or spent <= len(free):
                        take = free[spent - need:spent]
                        if copy:
                            self.refs[self.rows[s][-1]] -= 1
                            copies.append((self.rows[s].pop(), take[0], rest))
                        self.rows[s] += take
                        for g in take:
                            self.refs[g] = 1
                        self.lens[s] += n
                        give = n
                    else:
                        self.starved += 1
            granted.append(give)
        return granted, copies

    def drop(self, slots, n_drop):
        for s, n in zip(slots, n_drop):
            if s < 0:
                continue
            if s >= len(self.lens) or slots.count(s) > 1 or n < 0:
                self.faults += 1
                continue
            self.lens[s] = max(0, self.lens[s] - n)
            while len(self.rows[s]) > self.pages(self.lens[s]):
                self.refs[self.rows[s].pop()] -= 1

    def compact(self):
        n_live = sum(r != 0 for r in self.refs)
        remap = [g if r else -1 for g, r in enumerate(self.refs)]
        holes = [g for g in range(n_live) if self.refs[g] == 0]
        moves = []
        for g in range(n_live, len(self.refs)):
            if self.refs[g]:
                remap[g] = holes.pop(0)
                self.refs[remap[g]], self.refs[g] = self.refs[g], 0
                moves.append((g, remap[g]))
        self.rows = [[remap[g] for g in row] for row in self.rows]
        return remap, n_live, moves

    def matches(self, cache):
        table, lens, refs = cache.table.tolist(), cache.lens.tolist(), cache.refs.tolist()
        assert lens == self.lens
        assert refs == self.refs
        for s, row in enumerate(self.rows):
            assert table[s][:len(row)] == row, s


def u32(t):
    return torch.tensor(t, dtype=torch.int32, device="cuda")


def attention(cache, layer, Q, slots, n_new, scale=0.0):
    """O and A = sum_j p_j |v_j| in fp64, from the definition; cache has pool, table and lens tensors."""
    B, H, q_len, D = Q.shape
    page, KV = cache.page, cache.n_kv_heads
    O = torch.zeros((B, H, q_len, D), dtype=torch.float64, device=Q.device)
    A = torch.zeros_like(O)
    lens = cache.lens.tolist()
    for b, s in enumerate(slots):
        if s < 0:
            continue
        n = lens[s]
        at = torch.arange(n, device=Q.device)
        g, off = cache.table[s].long()[at // page], at % page
        k = cache.pool[2 * layer, g, :, off].double()   # [n, KV, D]
        v = cache.pool[2 * layer + 1, g, :, off].double()
        for i in range(n_new[b]):
            e = n - n_new[b] + i + 1
            if e <= 0:
                continue
            q = Q[b, :, i].double().reshape(KV, H // KV, D)
            x = torch.einsum("kgd,nkd->kgn", q, k[:e]) * (scale if scale > 0 else 1.0 / math.sqrt(D))
            w = torch.softmax(x, -1)
            O[b, :, i] = torch.einsum("kgn,nkd->kgd", w, v[:e]).reshape(H, D)
            A[b, :, i] = torch.einsum("kgn,nkd->kgd", w, v[:e].abs()).reshape(H, D)
    return O, A


def check_attention(O, want, A, n_keys, vmax):
    """Bound of |O - want|, element by element, with u the unit roundoff of the type (half a unit in the last
    place: 2^-8 for bf16's 8 significant bits, 2^-11 for fp16's 11): the rounding of O, u |O|; the rounding of the
    softmax numerators, u A; logits summed in fp32 over at most 128 products and the fast exponential, 2^-10 A
    for logits whose products add up to a few tens; and in fp16 numerators below the normal range, 2^-25 each
    against a sum of at least 1."""
    bf16 = O.dtype is torch.bfloat16
    u = 2.0 ** -8 if bf16 else 2.0 ** -11
    tol = u * want.abs() + (u + 2.0 ** -10) * A + (0.0 if bf16 else n_keys * 2.0 ** -25 * vmax) + 1e-7
    got = O.double()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol
    assert float(over.max()) <= 0.0, f"worst excess {float(over.max()):.3e}, error {float((got - want).abs().max()):.3e}"


def verify(p, q, draft, n_draft, ua, us):
    """The rule of wise_verify_draft on numpy arrays: p [B, K+1, V], q [B, K, V] as fp32 values."""
    B, K1, V = p.shape
    accepted, tokens = [], []

    def weights(r):
        r = np.where(np.isnan(r), np.float32(0), r).astype(np.float64)
        return [int(x) for x in np.floor(np.clip(r, 0.0, 1.0) * 2.0 ** 40)]

    for b in range(B):
        nd = K1 - 1 if n_draft is None else min(max(n_draft[b], 0), K1 - 1)
        n, out = 0, False
        while n < nd:
            x = int(draft[b][n])
            out = not 0 <= x < V
            if out or not np.float32(ua[b][n]) * q[b, n, x] < p[b, n, x]:
                break
            n += 1
        with np.errstate(invalid="ignore"):
            r = p[b, n] if n == nd or out else np.maximum(p[b, n] - q[b, n], np.float32(0))
        w = weights(r)
        if not any(w):
            w = weights(p[b, n])
        total, token = sum(w), -1
        if total:
            u = int(min(max(float(us[b]), 0.0), 1.0 - 2.0 ** -24) * 2 ** 24)
            t, run = total * u >> 24, 0
            for v, x in enumerate(w):
                run += x
                if run > t:
                    token = v
                    break
        accepted.append(n)
        tokens.append([int(x) for x in draft[b][:n]] + [token] + [-1] * (K1 - 1 - n))
    return accepted, tokens
