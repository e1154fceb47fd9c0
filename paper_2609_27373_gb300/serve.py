"""Answering with the model after its recurrent steps: a paged cache of keys
and values, attention of new tokens over it with shared prefixes, and the
verification of drafted tokens.

`PagedCache` keeps the device memory and the workspaces of one cache and calls
the library's entry points in their order of use:

    cache = PagedCache(n_layers=4, n_pages=4096, n_kv_heads=8, page=64, head_dim=128, n_slots=64, max_pages=512)
    cache.extend(slots, n_new)                      # room for a prompt's tokens (or each step's)
    cache.write(layer, slots, granted, K, V)        # each layer's keys and values, as they are computed
    cache.fork(src, dst)                            # samples of one prompt: pages are shared, not copied
    cache.attend(layer, Q, O, slots, granted, group_start, prefix_lens)
    accepted, tokens = verify_draft(p, q, draft, n_draft, u_accept, u_sample)
    cache.drop(slots, n_rejected)                   # rejected drafts, or sequences that ended
    cache.compact()                                 # pages in use to the front of the pool

Every call is asynchronous on `stream` (default: torch's current stream);
calls on one cache must be ordered on a stream, and two calls that may run at
the same time need a PagedCache each over the same tensors (`over`), since
each keeps one workspace.  Calls can be captured in a CUDA graph, for one shape
after another; the cache must outlive the graphs.  The cache's own memory is recorded on every stream
that its calls run on, so that the cache can be let go while they run; what a
call is given besides (lists, keys and values, queries, outputs) is the
caller's to keep.
"""
from __future__ import annotations

import torch

from . import wise


def _empty(shape, dtype, device, stream):
    """Memory of the stream that the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class PagedCache(wise.Cache):
    """A paged cache with its workspaces (see wise.Cache for the tensors)."""

    def __init__(self, n_layers: int, n_pages: int, n_kv_heads: int, page: int, head_dim: int, n_slots: int,
                 max_pages: int, dtype=torch.bfloat16, device=None):
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self._own(torch.empty((2 * n_layers, n_pages, n_kv_heads, page, head_dim), dtype=dtype, device=dev),
                  torch.zeros((n_slots, max_pages), dtype=torch.int32, device=dev),
                  torch.zeros((n_slots,), dtype=torch.int32, device=dev),
                  torch.zeros((n_pages,), dtype=torch.int32, device=dev))

    @classmethod
    def over(cls, pool, table, lens, refs) -> "PagedCache":
        """A cache over tensors that the caller holds."""
        cache = cls.__new__(cls)
        cache._own(pool, table, lens, refs)
        return cache

    def _own(self, pool, table, lens, refs) -> None:
        wise.Cache.__init__(self, pool, table, lens, refs)
        self._streams = {}     # streams that have used the cache, by handle
        self._workspaces = []  # all of them, see _grown
        self._kv_ws = None
        self._kv_n = -1
        self._attn_ws = None
        self._attn_key = self._attn_shape = None

    def _use(self, stream) -> int:
        """Before a call on `stream`: torch does not hand the cache's memory out again before that stream is done.
        Returns the stream's handle."""
        raw = wise._raw_stream(stream, self.index)
        if raw not in self._streams:
            self._streams[raw] = torch.cuda.current_stream(self.device) if stream is None else stream
            for t in (self.pool, self.table, self.lens, self.refs, *self._workspaces):
                t.record_stream(self._streams[raw])
        return raw

    def _grown(self, ws, need: int, stream):
        """The workspace `ws`, or a new one where `need` is more than it has.  A captured graph goes on writing to the
        one it was captured with, so none is given back before the cache is; each new one is at least twice as
        large, so that all the old ones together are no larger than the last."""
        have = 0 if ws is None else ws.numel()
        if ws is None or need > have:
            # 0 bytes: the library refuses this cache, and the call itself says why.
            ws = _empty(max(need, 2 * have, 16), torch.uint8, self.device, stream)
            self._workspaces.append(ws)
            for s in self._streams.values():
                ws.record_stream(s)
        return ws

    def _kv_workspace(self, n: int, stream):
        if n > self._kv_n:
            self._kv_ws = self._grown(self._kv_ws, wise.wise_kv_workspace(self, n), stream)
            self._kv_n = n
        return self._kv_ws

    def fork(self, src, dst, stream=None) -> None:
        """Slots dst[i] become forks of slots src[i]; pages are shared until one of the holders grows."""
        wise.wise_kv_fork(self, src, dst, self._use(stream))

    def extend(self, slots, n_new, granted=None, stream=None):
        """Grows the sequences by n_new tokens each; returns what was granted (n_new, or 0 where pages ran out)."""
        raw = self._use(stream)
        if granted is None:
            granted = _empty(n_new.shape, torch.int32, self.device, stream)
        wise.wise_kv_extend(self, slots, n_new, granted, self._kv_workspace(slots.shape[0], stream), raw)
        return granted

    def write(self, layer: int, slots, granted, K, V, stream=None) -> None:
        """Stores one layer's new keys and values [batch, n_kv_heads, q_len, head_dim] at the sequences' ends."""
        wise.wise_kv_write(self, layer, slots, granted, K, V, self._use(stream))

    def drop(self, slots, n_drop, stream=None) -> None:
        """Takes the last n_drop tokens (at most all) off each sequence."""
        wise.wise_kv_drop(self, slots, n_drop, self._use(stream))

    def compact(self, stream=None):
        """Moves the pages in use to the front of the pool; returns remap int32 [n_pages] and n_live int32 [1]."""
        raw = self._use(stream)
        remap = _empty(self.n_pages, torch.int32, self.device, stream)
        n_live = _empty(1, torch.int32, self.device, stream)
        wise.wise_kv_compact(self, remap, n_live, self._kv_workspace(0, stream), raw)
        return remap, n_live

    def attend(self, layer: int, Q, O, slots, n_new=None, group_start=None, prefix_lens=None, scale: float = 0.0,
               stream=None) -> None:
        """Attention of Q [batch, n_heads, q_len, head_dim] over the sequences in slots, into O; the requests of
        each group share their first prefix_lens[g] tokens."""
        raw = self._use(stream)
        key = (Q.shape, 0 if prefix_lens is None else prefix_lens.shape[0], scale)
        if key != self._attn_key:
            shape = wise.prefix_shape(self, Q, key[1], scale)
            self._attn_ws = self._grown(self._attn_ws, wise.wise_prefix_attn_workspace(self, shape), stream)
            self._attn_key, self._attn_shape = key, shape
        wise.wise_prefix_attn(self, layer, Q, O, slots, n_new, group_start, prefix_lens, self._attn_ws, scale, raw,
                              self._attn_shape)


def verify_draft(p, q, draft, n_draft, u_accept, u_sample, stream=None):
    """Verifies drafted tokens; returns accepted int32 [batch] and tokens int32 [batch, k + 1] (the accepted tokens,
    the next token, then -1)."""
    accepted = _empty(p.shape[0], torch.int32, p.device, stream)
    tokens = _empty((p.shape[0], p.shape[1]), torch.int32, p.device, stream)
    wise.wise_verify_draft(p, q, draft, n_draft, u_accept, u_sample, accepted, tokens, stream)
    return accepted, tokens
