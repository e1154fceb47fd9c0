// The attention kernel of prefix_attn.cuh, one instance per head dimension and
// 16-bit type.
//
// Warp roles (384 threads):
//   warps 0-3, 4-7  softmax of stream 0 and 1: thread t of a warpgroup owns
//                   query row t (TMEM lane t).  Reads S from tensor memory,
//                   masks, keeps the row's running maximum and sum in fp32,
//                   writes P as 16-bit pairs, rescales O when the maximum
//                   moved by more than 2^8, and at the end of a segment stores
//                   (m, l) and O to the workspace.  Warps without a query row
//                   only keep the barriers going.
//   warps 8, 11     producers: walk the tiles of stream 0 and 1, look their
//                   pages up (a lane per page, one tile ahead), publish the
//                   schedule and issue the TMA loads of Q, K and V.
//   warp 9          one thread: S = Q K^T of both streams in turn.
//   warp 10         one thread: O += P V of both streams in turn.
// TMEM: S at column 0, P of stream w at 128 + 64 w, O at 256 + 128 w; with a
// head dimension of 64 there is room for an S of each stream (stream 1's at
// 384, O at 256 + 64 w).  S is handed to the next product as soon as it has
// been read, so a stream's softmax runs beside the products of the other one
// and beside its own next S.  (With P written over S, and one issuing thread a
// stream, the next S had to wait for P V: 5250 clk a pair's tile of 128 + 128
// rows at head dimension 128; now 3700, two turns of the one S buffer: 8
// products at 89 clk, 400 until the softmax sees S, 300 to read it, 380 until
// the next product.)
//
// What bounds it.  Long unshared sequences: HBM (38 x 8 x 8001 tokens of 128,
// 1.25 GB, in 181 us, 6.9 TB/s).  Middling ones (64 x 1001 tokens, 53 us, floor
// 39; 16 requests on a prefix of 4096, 32.5 us, floor 16) have too few tiles to
// make up for the start, the merge and, at head dimensions 96 and 128, the one K
// and one V slot of a stream that works alone.  Prefixes with 256 or more query rows a kv
// head: the S buffer, at about half of the tensor rate.  Short items: one
// warp's softmax of a tile (3600 to 4200 clk, twice what its instructions would
// take if they were at hand) in 7000 clk from tile to tile.  So S is read whole
// and given back before it is masked: with masked tiles taken 32 columns at a
// time the other stream waited for S (256 samples on a prefix of 8192 tokens:
// 74 us, now 71).  Small calls: the first microseconds of a launch, in which
// every line of code comes from far away.
//
// Every wait is bounded; one that runs out sets the status word and an abort
// flag, and every role unwinds.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_common.cuh"
#include "prefix_attn.cuh"
#include "ptx.cuh"

namespace wise {

template <int D>
struct PfxCfg {
  static constexpr int kBoxes = (D + 63) / 64;
  static constexpr int kTileBytes = kBoxes * 128 * 128;  // a Q, K or V tile
  static constexpr int kSlots = 64 * 1024 / kTileBytes;  // of the K ring and of the V ring: 64 KB each
  static constexpr int kThreads = 384;
  static constexpr int kRegsSoftmax = 208;  // 256 * 208 + 128 * 88 <= 384 * 168 registers
  static constexpr int kRegsOther = 88;
  static constexpr int kRingBytes = (2 + 2 * kSlots) * kTileBytes;  // two Q tiles, then the rings
  static constexpr int kMaxPlanBytes = 33 * 1024;
  static constexpr int kSBufs = D == 64 ? 2 : 1;
  static constexpr uint32_t kTmemP = 128, kTmemO = 256;
  static constexpr uint32_t kTmemOStep = D == 64 ? 64 : 128;
  static constexpr uint32_t kTmemS1 = 384;
  static constexpr int kSmemFixed = kRingBytes + 1024;  // and the plan behind
  static_assert(kSmemFixed + kMaxPlanBytes + 1024 <= 227 * 1024, "shared memory");
  static_assert(256 * kRegsSoftmax + 128 * kRegsOther <= kThreads * 168, "register split");
};

constexpr int kPfxSched = 8;  // schedule entries per stream
constexpr int kPfxFirst = 1, kPfxLast = 2, kPfxEnd = 4, kPfxFaulty = 8;

// Schedule entry {ring slot | parity of its use << 8 | keys << 16, first key position,
// request | (requests - 1) << 10 | kind << 17 | flags << 19, segment slot}.
__device__ __forceinline__ int pfx_pack(int req, int nreq, int kind, int flags) {
  return req | (nreq - 1) << 10 | kind << 17 | flags << 19;
}

template <int NS>
struct PfxShared {
  uint64_t k_full[NS], k_empty[NS], v_full[NS], v_empty[NS];
  uint64_t sched_full[2][kPfxSched], sched_empty[2][kPfxSched];  // empty: the two issuers and 4 warps
  uint64_t q_full[2], q_free[2];
  uint64_t s_full[2];  // S of a stream written
  uint64_t s_free[2];  // S buffer read: 4 warps
  uint64_t p_full[2];  // P written (and O read where a segment ended): 4 warps
  uint64_t o_full[2];  // P V completed
  uint64_t done[2];
  int4 sched[2][kPfxSched];
  uint32_t tmem_base;
  int abort;
};

// ---------------------------------------------------------------------- plan
// Written for few instructions: in a launch's first microseconds every line of
// code is fetched from far away (some 500 clk for 8 instructions).
// All threads of the CTA; `plan` in shared memory.
__device__ inline void pfx_make_plan(const PfxParams& p, const PfxPlan& plan, bool report) {
  const CacheView& c = p.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
  int bad = 0, bad_groups = 0;
#pragma unroll 1
  for (int g = tid; g <= p.n_groups; g += blockDim.x) {
    if (p.n_groups == 0) break;
    const int a = p.group_start[g], e = g < p.n_groups ? p.group_start[g + 1] : a;
    if (g < p.n_groups) plan.tiles[g] = p.prefix_lens[g];  // the declared length, until the tiles are known
    if (a < 0 || a > p.batch || a > e) bad_groups = 1;
    plan.start[g] = a;
  }
#pragma unroll 1
  for (int r = tid; r < p.batch; r += blockDim.x) {
    const int s = p.slots[r];
    const int add = p.n_new ? p.n_new[r] : p.q_len;
    int len = 0;
    if (s >= 0) {
      len = s < c.n_slots ? c.lens[s] : -1;
      if (len < 0 || len > c.max_len || add < 0 || add > p.q_len) {
        bad = 1;
        len = 0;
      }
    }
    plan.slot[r] = s;
    plan.len[r] = add > 0 ? len : 0;
    plan.add[r] = add > 0 ? add : 0;
    plan.lo[r] = 0;
    plan.group[r] = -1;
  }
  if (report && (bad | bad_groups)) atomicOr(c.status, kStatusBadCache);
  const bool grouped = !__syncthreads_or(bad_groups);
#pragma unroll 1
  for (int g = warp; g < p.n_groups; g += n_warps) {
    const int a = plan.start[g], e = plan.start[g + 1];
    int shortest = INT_MAX, active = 0, lead = INT_MAX;
    if (grouped) {
#pragma unroll 1
      for (int r = a + lane; r < e; r += 32) {
        const int len = plan.len[r];
        if (len > 0) {
          shortest = min(shortest, len);
          lead = min(lead, r);
          ++active;
        }
      }
    }
    shortest = __reduce_min_sync(0xffffffffu, shortest);
    active = __reduce_add_sync(0xffffffffu, active);
    lead = __reduce_min_sync(0xffffffffu, lead);
    int shared = 0;
    if (active > 1) shared = max(0, min(plan.tiles[g], shortest)) & -c.page;
    __syncwarp();
    const int tiles = (shared + kPfxKeys - 1) / kPfxKeys;
    if (lane == 0) {
      plan.tiles[g] = tiles;
      plan.lead[g] = lead;
      const int row_tiles = tiles > 0 ? (e - a + p.per_tile - 1) / p.per_tile : 0;
      const int pairs = row_tiles >> 1, single = row_tiles & 1;
      plan.pairs[g] = pairs;
      plan.pair_base[g] = pairs * tiles * c.n_kv_heads;
      plan.pair_item[g] = pairs;
      plan.single_base[g] = single * tiles * c.n_kv_heads;
      plan.single_item[g] = single;
    }
    if (shared > 0) {
#pragma unroll 1
      for (int r = a + lane; r < e; r += 32) {
        plan.lo[r] = shared;
        plan.group[r] = g;
      }
    }
  }
  __syncthreads();
  // Prefix sums, a warp each, four entries a lane: the groups' four counts
  // (warps 0-3) and the requests' own tiles (warp 4).
  if (warp < 5) {
    int* list = warp < 4 ? plan.pair_base + warp * (p.n_groups + 1) : plan.cum;
    const int n = warp < 4 ? p.n_groups : p.batch;
    int before = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += 128) {
      const int first = i0 + 4 * lane;
      int x[4], sum = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = 0;
        if (first + k < n)
          x[k] = warp < 4 ? list[first + k]
                          : max(0, plan.len[first + k] - plan.lo[first + k] + kPfxKeys - 1) / kPfxKeys;
        sum += x[k];
      }
      int upto = sum;
#pragma unroll 1
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
      }
      int at = before + upto - sum;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (first + k < n) list[first + k] = at;
        at += x[k];
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) list[n] = before;
  }
  __syncthreads();
  if (tid < 2) {  // thread 0 cuts the line of pair items, thread 1 the other one
    const int single = plan.single_base[p.n_groups];
    const PfxCuts cuts = pfx_cuts(tid == 0 ? plan.pair_base[p.n_groups] : single + plan.cum[p.batch] * c.n_kv_heads,
                                  gridDim.x << tid);
    (tid == 0 ? plan.t->pair : plan.t->line) = cuts;
    if (tid == 0) plan.t->single_tiles = single;
  }
  __syncthreads();
}

// Largest g with base[g] <= x (base ascending, base[0] <= x < base[n]).
__device__ __forceinline__ int pfx_find(const int* base, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (base[mid] <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Waits of the producers and issuers: the polling loop is one function, which
// keeps their own loops short.  (The softmax has no registers for a call.)
static __device__ __noinline__ bool pfx_wait_long(uint64_t* bar, uint32_t parity, volatile int* abort,
                                                  uint64_t limit_ns) {
  return mbar_wait(bar, parity, abort, limit_ns);
}
__device__ __forceinline__ bool pfx_wait(uint64_t* bar, uint32_t parity, volatile int* abort, uint64_t limit_ns) {
  return mbar_try_wait(bar, parity) || pfx_wait_long(bar, parity, abort, limit_ns);
}
__device__ __forceinline__ bool pfx_warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort, uint64_t limit_ns) {
  return __all_sync(0xffffffffu, pfx_wait(bar, parity, abort, limit_ns));
}
// A wait ran out: every role unwinds.
static __device__ __noinline__ void pfx_give_up(int* abort, int* status) {
  *reinterpret_cast<volatile int*>(abort) = 1;
  atomicOr(status, kStatusTimeout);
}

// The row of the tile at which an own item's rows start.  Few rows keep one
// warp of a stream busy; that of stream 1 is then on another scheduler of the
// SM than that of stream 0 (256 samples on a prefix of 8192 tokens: 72.8 us on
// the same scheduler, 71.0 on any other one; 64 requests on one of 32768: 72.2 and
// 71.1; 2432 items of one row and one tile: 42.7 and 42.4; the few rows of prefix
// items gain nothing from it).
__device__ __forceinline__ int pfx_own_row(const PfxParams& p, int w) { return w == 1 && p.rows <= 32 ? 96 : 0; }

// A segment: a run of key tiles of an item.
struct PfxSeg {
  int word, word2;  // requests and kind as in a schedule entry; of a pair's second tile
  int kvh, row;     // kv head, cache slot whose pages are read
  int pos, end;     // position of the next tile's first key; one past the item's keys
  int left;         // tiles left
  int slot;         // workspace slot
};

// The segment that starts at tile x of a line and ends at x_end or with its item.
__device__ __forceinline__ PfxSeg pfx_segment(const PfxParams& p, const PfxPlan& plan, bool pairs, int x, int x_end,
                                              int run) {
  PfxSeg s;
  const int kv = p.cache.n_kv_heads;
  const int single_tiles = plan.t->single_tiles;
  int tiles, t, kind, nreq, nreq2 = 1, req;
  if (pairs || x < single_tiles) {
    const int* base = pairs ? plan.pair_base : plan.single_base;
    const int g = pfx_find(base, p.n_groups, x);
    tiles = plan.tiles[g];
    const int y = x - base[g];
    const int it = y / tiles;
    t = y - it * tiles;
    const int a = plan.start[g], members = plan.start[g + 1] - a;
    const int n_pairs = plan.pairs[g];
    if (pairs) {
      // kv head outermost: the pairs of one kv head read the same keys at about the same time.
      s.kvh = it / n_pairs;
      const int pair = it - s.kvh * n_pairs;
      kind = kPfxPair;
      req = a + 2 * pair * p.per_tile;
      s.slot = 2 * (plan.pair_item[g] * kv + it + run);
      nreq = p.per_tile;
      nreq2 = min(p.per_tile, members - (2 * pair + 1) * p.per_tile);
    } else {
      s.kvh = it;
      kind = kPfxSingle;
      req = a + 2 * n_pairs * p.per_tile;  // the odd tile is the last one
      s.slot = plan.single_item[g] * kv + it + run;
      nreq = members - 2 * n_pairs * p.per_tile;
    }
    const int lead = plan.lead[g];
    s.row = plan.slot[lead];
    s.end = plan.lo[lead];
    s.pos = t * kPfxKeys;
  } else {
    const int y = x - single_tiles;
    // cum[r] * kv <= y < cum[r + 1] * kv
    req = pfx_find(plan.cum, p.batch, y / kv);
    tiles = plan.cum[req + 1] - plan.cum[req];
    const int z = y - plan.cum[req] * kv;
    s.kvh = z / tiles;
    t = z - s.kvh * tiles;
    kind = kPfxOwn;
    nreq = 1;
    s.row = plan.slot[req];
    s.end = plan.len[req];
    s.pos = plan.lo[req] + t * kPfxKeys;
    s.slot = req * kv + s.kvh + run;
  }
  s.left = min(tiles - t, x_end - x);
  s.word = pfx_pack(req, nreq, kind, 0);
  s.word2 = pairs ? pfx_pack(req + p.per_tile, nreq2, kind, 0) : 0;
  return s;
}

// Tiles of run k of a line (0 past its last run).
__device__ __forceinline__ int pfx_run_tiles(const PfxCuts& c, int k) {
  return k < c.runs ? pfx_cut(c, k + 1) - pfx_cut(c, k) : 0;
}

// ----------------------------------------------------------------- producers
// The items of the second line come first, then the pair items: their partial
// results, the larger ones, are then still in L2 when the merge reads them.
//
// Ring slots.  At first stream w has the slots w * NS / 2 .. of each ring to
// itself.  While pair items run, tile n of them sits in slot n % NS of both
// rings and both streams use it.  A slot's uses are counted across both
// phases: use u waits for the end of use u - 1.

// One warp each: warp 8 (w = 0) and warp 11 (w = 1).  Each publishes the
// schedule and loads Q of its stream, and at first its K and V tiles; while
// pair items run, warp 8 loads the K tiles and warp 11 the V tiles of both.
template <int D>
__device__ void pfx_producer(const CUtensorMap* mapK, const CUtensorMap* mapV, const CUtensorMap* mapQ,
                             const CUtensorMap* mapQ1, const PfxParams& p, const PfxPlan& plan, int w,
                             uint8_t* q_tiles, uint8_t* ring, PfxShared<PfxCfg<D>::kSlots>& sb) {
  using C = PfxCfg<D>;
  constexpr int NS = C::kSlots, H = NS / 2;
  const CacheView& c = p.cache;
  const int lane = threadIdx.x & 31;
  volatile int* abort = &sb.abort;
  const PfxTotals t = *plan.t;
  const int cta = blockIdx.x;
  // Runs of the line start at the CTA after the last one with pair items, so
  // that small problems spread out.
  int line_run = cta - t.pair.runs;
  if (line_run < 0) line_run += gridDim.x;
  const int n0 = pfx_run_tiles(t.line, line_run), n1 = pfx_run_tiles(t.line, line_run + gridDim.x);
  line_run += w * gridDim.x;
  int n_ent = 0, n_q = 0;            // schedule entries published, Q tiles loaded
  uint32_t issued = 0, parity = 0;   // by ring (8 bits each) and slot: loads of this warp, and their last use's parity
  int bad = 0;
  bool ok = true;

  const bool has_pairs = cta < t.pair.runs;
  bool pair = false;
  int run = line_run;
  int x = pfx_cut(t.line, run), x_end = x + (w ? n1 : n0);
  int n = 0;  // tiles of the phase so far
  PfxSeg seg;
  seg.left = 0;
  int page = -1;       // this lane's page of the next tile, not looked at before its turn
  bool first = false;  // the next tile starts its segment

  auto fetch = [&]() {
    const int at = seg.pos + (lane << c.page_shift);
    page = -1;
    if (at - seg.pos < kPfxKeys && at < seg.end)
      page = __ldg(c.table + (size_t)seg.row * c.max_pages + (at >> c.page_shift));
  };
  for (;;) {
    if (seg.left == 0) {
      if (x == x_end) {
        if (pair || !has_pairs) break;
        // Both warps have issued all loads of the first phase when they go on:
        // the other's slots are then at most one use behind, which is as far
        // as a wait can tell.
        named_barrier_sync(1, 64);
        pair = true;
        n = 0;
        run = cta;
        x = pfx_cut(t.pair, run);
        x_end = pfx_cut(t.pair, run + 1);
      }
      seg = pfx_segment(p, plan, pair, x, x_end, run);
      x += seg.left;
      first = true;
      fetch();
    }
    const bool second = pair && w == 1;
    const int slot = pair ? n % NS : w * H + n % H;
    const int use = pair ? n / NS + ((slot < H ? n0 : n1) - slot % H + H - 1) / H : n / H;
    const int word = second ? seg.word2 : seg.word;
    // The lane's page of the tile, if the item reaches it.
    const int at = lane << c.page_shift;
    const bool on = at < kPfxKeys && seg.pos + at < seg.end;
    const bool valid = page >= 0 && page < c.n_pages;
    const bool faulty = __any_sync(0xffffffffu, on && !valid);
    if (faulty) bad = 1;
    const int e = n_ent % kPfxSched;
    if (n_ent >= kPfxSched) ok = pfx_warp_wait(&sb.sched_empty[w][e], ((n_ent / kPfxSched) - 1) & 1, abort, p.wait_ns);
    if (ok && lane == 0) {
      const int flags = (first ? kPfxFirst : 0) | (seg.left == 1 ? kPfxLast : 0) | (faulty ? kPfxFaulty : 0);
      sb.sched[w][e] = make_int4(slot | (use & 1) << 8 | min(kPfxKeys, seg.end - seg.pos) << 16, seg.pos,
                                 word | flags << 19, seg.slot + second);
      mbar_arrive(&sb.sched_full[w][e]);
    }
    ++n_ent;
    // The tile of the K ring (r = 0) and of the V ring; Q in between.  A faulty
    // page id becomes a coordinate out of range, which reads zeros.
    const int z = valid ? page * c.n_kv_heads + seg.kvh : c.n_pages * c.n_kv_heads;
    const int bytes = min(kPfxKeys, (seg.end - seg.pos + c.page - 1) & -c.page) * 128 * C::kBoxes;
#pragma unroll 1
    for (int r = pair ? w : 0; ok && r <= (pair ? w : 1); ++r) {
      uint64_t* full = r ? &sb.v_full[slot] : &sb.k_full[slot];
      uint64_t* empty = r ? &sb.v_empty[slot] : &sb.k_empty[slot];
      if (use >= 1) ok = pfx_warp_wait(empty, (use - 1) & 1, abort, p.wait_ns);
      if (!ok) break;
      if (lane == 0) mbar_arrive_expect_tx(full, bytes);
      __syncwarp();
      if (on) {
        uint8_t* dst = ring + (r * NS + slot) * C::kTileBytes + at * 128;
#pragma unroll
        for (int b = 0; b < C::kBoxes; ++b)
          tma_load_3d(dst + b * 128 * 128, r ? mapV : mapK, full, 64 * b, 0, z);
      }
      const uint32_t bit = 1u << (r * 8 + slot);
      issued |= bit;
      parity = (use & 1) ? parity | bit : parity & ~bit;
      if (first) {
        first = false;
        if (n_q >= 1) ok = pfx_warp_wait(&sb.q_free[w], (n_q - 1) & 1, abort, p.wait_ns);
        if (!ok) break;
        if (lane == 0) {
          const bool own = ((word >> 17) & 3) == kPfxOwn;
          mbar_arrive_expect_tx(&sb.q_full[w], (own ? p.rows : p.rows * p.per_tile) * 128 * C::kBoxes);
#pragma unroll
          for (int b = 0; b < C::kBoxes; ++b)
            tma_load_4d(q_tiles + w * C::kTileBytes + (b * 128 + (own ? pfx_own_row(p, w) : 0)) * 128,
                        own ? mapQ1 : mapQ, &sb.q_full[w], 64 * b, 0, seg.kvh, word & 1023);
        }
        ++n_q;
      }
    }
    if (!ok) break;
    ++n;
    --seg.left;
    seg.pos += kPfxKeys;
    if (seg.left > 0) fetch();
  }
  if (has_pairs && !pair) named_barrier_sync(1, 64);  // gave up in the first phase
  if (ok) {
    const int e = n_ent % kPfxSched;
    if (n_ent >= kPfxSched) ok = pfx_warp_wait(&sb.sched_empty[w][e], ((n_ent / kPfxSched) - 1) & 1, abort, p.wait_ns);
    if (ok && lane == 0) {
      sb.sched[w][e] = make_int4(0, 0, kPfxEnd << 19, 0);
      mbar_arrive(&sb.sched_full[w][e]);
    }
  }
  if (bad && lane == 0) atomicOr(c.status, kStatusBadCache);
  if (!ok && lane == 0) {
    pfx_give_up(&sb.abort, c.status);
    // Copies already issued land before the CTA's shared memory is released.
    int never = 0;
    for (int k = 0; k < NS; ++k) {
      if ((issued >> k) & 1) mbar_wait(&sb.k_full[k], (parity >> k) & 1, &never);
      if ((issued >> (8 + k)) & 1) mbar_wait(&sb.v_full[k], (parity >> (8 + k)) & 1, &never);
    }
    if (n_q > 0) mbar_wait(&sb.q_full[w], (n_q - 1) & 1, &never);
  }
  __syncwarp();
}

// --------------------------------------------------------------- MMA issuers
// Both issuing threads take the streams in turn, tile by tile, until a stream
// ends.  The streams' runs have equally many tiles up to one, so the fixed
// order costs little; threads that poll both streams and take whichever is
// ready load the shared-memory pipe so much that every other wait of the SM
// slows down (94 us instead of 74 for 64 requests on a 32K prefix).
struct PfxTurn {
  int j;     // tile
  int nq;    // segments started
  bool end;
};

template <bool FP16>
__device__ __forceinline__ constexpr uint32_t pfx_idesc(uint32_t bf16) {
  return FP16 ? bf16 & ~((1u << 7) | (1u << 10)) : bf16;  // operand type 0: fp16, 1: bf16
}

// One thread: the S products.  (The two streams share one copy of the code, as
// everywhere in this kernel: its loops together stay small enough for the
// instruction cache, whose misses bounded larger variants.)
template <int D, bool FP16>
__device__ void pfx_mma_s(const PfxParams& p, int second, uint32_t tmem, uint8_t* q_tiles, uint8_t* ring,
                          PfxShared<PfxCfg<D>::kSlots>& sb) {
  using C = PfxCfg<D>;
  volatile int* abort = &sb.abort;
  constexpr uint32_t idesc = pfx_idesc<FP16>(idesc_bf16_f32(128, kPfxKeys, false, false));
  constexpr bool own_buf = C::kSBufs == 2;
  PfxTurn t = {}, other = {};  // this turn's stream and the other one
  int used = 0, used_other = 0;  // uses of the stream's S buffer
  bool ok = true;
#pragma unroll 1
  for (int w = 0; !(t.end && other.end); w ^= 1) {
    if (!t.end) {
      const int e = t.j % kPfxSched;
      if (!pfx_wait(&sb.sched_full[w][e], (t.j / kPfxSched) & 1, abort, p.wait_ns)) {
        ok = false;
        break;
      }
      const int4 ent = sb.sched[w][e];
      mbar_arrive(&sb.sched_empty[w][e]);
      const int flags = ent.z >> 19, slot = ent.x & 255;
      if (flags & kPfxEnd) {
        t.end = true;
      } else {
        if (((flags & kPfxFirst) && !pfx_wait(&sb.q_full[w], t.nq++ & 1, abort, p.wait_ns)) ||
            !pfx_wait(&sb.k_full[slot], (ent.x >> 8) & 1, abort, p.wait_ns) ||
            (used > 0 && !pfx_wait(&sb.s_free[own_buf ? w : 0], (used - 1) & 1, abort, p.wait_ns))) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
        const uint64_t q0 = smem_desc_sw128(smem_u32(q_tiles + w * C::kTileBytes), 16, 1024);
        const uint64_t k0 = smem_desc_sw128(smem_u32(ring + slot * C::kTileBytes), 16, 1024);
        const uint32_t s_col = tmem + (own_buf && w == 1 ? C::kTmemS1 : 0);
        uint32_t acc = 0;
#pragma unroll 1
        for (int kk = 0; kk < D / 16; kk += 2) {  // 32 columns at a time
          const uint32_t off = ((kk >> 2) * (128 * 128) + (kk & 2) * 32) >> 4;
          umma_ss_split(s_col, (uint32_t)q0 + off, (uint32_t)(q0 >> 32), (uint32_t)k0 + off, (uint32_t)(k0 >> 32), idesc,
                        acc);
          acc = 1;
          umma_ss_split(s_col, (uint32_t)q0 + off + 2, (uint32_t)(q0 >> 32), (uint32_t)k0 + off + 2,
                        (uint32_t)(k0 >> 32), idesc, acc);
        }
        umma_commit(&sb.s_full[w]);
        // A commit covers every product of this thread before it, so a pair's
        // slot is given back with the second of its two products.
        if (((ent.z >> 17) & 3) != kPfxPair || w == second) umma_commit(&sb.k_empty[slot]);
        if (flags & kPfxLast) umma_commit(&sb.q_free[w]);
        ++used;
        ++t.j;
      }
    }
    const PfxTurn swap = t;
    t = other;
    other = swap;
    if (own_buf) {
      const int u = used;
      used = used_other;
      used_other = u;
    }
  }
  if (!ok) {
    pfx_give_up(&sb.abort, p.cache.status);
  }
  // Every MMA and commit of this thread completes before TMEM is released.
  umma_commit(&sb.done[0]);
  int never = 0;
  mbar_wait(&sb.done[0], 0, &never);
}

// One thread: the P V products.
template <int D, bool FP16>
__device__ void pfx_mma_pv(const PfxParams& p, int second, uint32_t tmem, uint8_t* ring, PfxShared<PfxCfg<D>::kSlots>& sb) {
  using C = PfxCfg<D>;
  constexpr int NS = C::kSlots;
  volatile int* abort = &sb.abort;
  constexpr uint32_t idesc = pfx_idesc<FP16>(idesc_bf16_f32(128, D, false, true));
  PfxTurn t = {}, other = {};
  bool ok = true;
#pragma unroll 1
  for (int w = 0; !(t.end && other.end); w ^= 1) {
    if (!t.end) {
      const int e = t.j % kPfxSched;
      if (!pfx_wait(&sb.sched_full[w][e], (t.j / kPfxSched) & 1, abort, p.wait_ns)) {
        ok = false;
        break;
      }
      const int4 ent = sb.sched[w][e];
      mbar_arrive(&sb.sched_empty[w][e]);
      const int flags = ent.z >> 19, slot = ent.x & 255;
      if (flags & kPfxEnd) {
        t.end = true;
      } else {
        if (!pfx_wait(&sb.v_full[slot], (ent.x >> 8) & 1, abort, p.wait_ns) ||
            !pfx_wait(&sb.p_full[w], t.j & 1, abort, p.wait_ns)) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
        const uint64_t v0 = smem_desc_sw128(smem_u32(ring + (NS + slot) * C::kTileBytes), kPfxKeys * 128, 1024);
        const uint32_t o_col = tmem + C::kTmemO + w * C::kTmemOStep, p_col = tmem + C::kTmemP + w * 64;
        uint32_t acc = (flags & kPfxFirst) ? 0u : 1u;
        const int steps = ((ent.x >> 16) + 15) / 16;  // of 16 keys; those past the item's end are left out
#pragma unroll 1
        for (int kk = 0; kk < steps; ++kk) {
          umma_ts_split(o_col, p_col + kk * 8, (uint32_t)v0 + kk * (2048 / 16), (uint32_t)(v0 >> 32), idesc, acc);
          acc = 1;
        }
        umma_commit(&sb.o_full[w]);
        if (((ent.z >> 17) & 3) != kPfxPair || w == second) umma_commit(&sb.v_empty[slot]);
        ++t.j;
      }
    }
    const PfxTurn swap = t;
    t = other;
    other = swap;
  }
  if (!ok) {
    pfx_give_up(&sb.abort, p.cache.status);
  }
  umma_commit(&sb.done[1]);
  int never = 0;
  mbar_wait(&sb.done[1], 0, &never);
}

// ------------------------------------------------------------------- softmax
template <bool FP16>
__device__ __forceinline__ uint32_t pack_16x2(float lo, float hi) {
  if constexpr (FP16) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  } else {
    return pack_bf16x2(lo, hi);
  }
}

template <int D, bool FP16>
__device__ void pfx_softmax(const PfxParams& p, const PfxPlan& plan, int w, uint32_t tmem, uint8_t* ring,
                            PfxShared<PfxCfg<D>::kSlots>& sb) {
  using C = PfxCfg<D>;
  constexpr int NS = C::kSlots;
  constexpr float kRescaleThreshold = 8.0f;  // log2 units: P stays <= 2^(8 + kLift)
  // P is rounded to the cache's type for the tensor cores (l is summed before).
  // fp16 ends at 2^-24, so its P are held 2^7 higher, at most 2^15: what is lost
  // is below 2^-32 of the row's largest a key.  (Without that 2^20 keys of 2^-26
  // each, 1.5 % of a row, vanished from the numerator.)
  constexpr float kLift = FP16 ? 7.0f : 0.0f;
  volatile int* abort = &sb.abort;
  const int r = threadIdx.x & 127, wq = r >> 5, lane = r & 31;
  const uint32_t lane_tmem = tmem + ((uint32_t)(wq * 32) << 16);
  constexpr bool own_buf = C::kSBufs == 2;
  const uint32_t s_col = own_buf && w == 1 ? C::kTmemS1 : 0, p_col = C::kTmemP + w * 64;
  const uint32_t o_col = C::kTmemO + w * C::kTmemOStep;
  uint64_t* s_free = &sb.s_free[own_buf ? w : 0];
  bool ok = true;
  // The thread's row of any tile: its request among the tile's, its new token.
  const int of = r / p.rows, i = (r - of * p.rows) % p.q_len;
  const int own_r = r - pfx_own_row(p, w), own_i = own_r < 0 ? 0 : own_r % p.q_len;
  int limit = 0;                                        // keys the row may see
  bool row_on = false, live = false, warp_on = false;  // a row of the item; one that sees keys; a warp with such
  float m = -INFINITY, l = 0.0f;
  for (int j = 0;; ++j) {
    const int e = j % kPfxSched;
    if (!warp_wait(&sb.sched_full[w][e], (j / kPfxSched) & 1, abort, p.wait_ns)) {
      ok = false;
      break;
    }
    const int4 ent = sb.sched[w][e];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sb.sched_empty[w][e]);
    const int flags = ent.z >> 19, kind = (ent.z >> 17) & 3;
    if (flags & kPfxEnd) break;
    if (flags & kPfxFirst) {
      const int req0 = ent.z & 1023, nreq = ((ent.z >> 10) & 127) + 1;
      const bool own = kind == kPfxOwn;
      row_on = own ? own_r >= 0 && own_r < p.rows : of < nreq;
      int seen = 0;
      if (row_on) {
        const int req = req0 + (own ? 0 : of), add = plan.add[req], k = own ? own_i : i;
        seen = k < add ? plan.len[req] - add + k + 1 : 0;
      }
      // Threads whose row sees nothing (or is none) compute on whatever Q
      // holds there and store no O; unmasked, they do not hold up their warp.
      live = seen > 0;
      limit = live ? seen : INT_MAX;
      warp_on = __any_sync(0xffffffffu, live);
      m = -INFINITY;
      l = 0.0f;
    }
    if (!warp_wait(&sb.s_full[w], j & 1, abort, p.wait_ns)) {
      ok = false;
      break;
    }
    tc_fence_after_sync();
    const int keys = ent.x >> 16;                        // of the tile
    const int lim = min(limit - ent.y, keys) - 1;        // last column the row sees
    const bool masked = __any_sync(0xffffffffu, lim < kPfxKeys - 1);
    float m_new = m, sum = 0.0f;
    uint32_t pw[kPfxKeys / 2];
    if (warp_on) {
      float s[kPfxKeys];
      tmem_load_row<kPfxKeys>(lane_tmem + s_col, s);
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_free);
      if (masked) {
#pragma unroll
        for (int c = 0; c < kPfxKeys / 32; ++c) {
          // Bit k: the row sees column 32 c + k.
          const int n = lim + 1 - 32 * c;
          const uint32_t seen = n >= 32 ? ~0u : n > 0 ? (1u << n) - 1 : 0u;
#pragma unroll
          for (int k = 0; k < 32; ++k) s[32 * c + k] = (seen >> k) & 1 ? s[32 * c + k] : -INFINITY;
        }
      }
      const float m_tile = row_max(s) * p.scale_log2 - kLift;
      m_new = (m_tile > m + kRescaleThreshold) ? m_tile : m;
      sum = exp2_scaled(s, p.scale_log2, m_new == -INFINITY ? 0.0f : m_new);
#pragma unroll
      for (int k = 0; k < kPfxKeys / 2; ++k) pw[k] = pack_16x2<FP16>(s[2 * k], s[2 * k + 1]);
    } else if (lane == 0) {
      mbar_arrive(s_free);
    }
    // P and O are at rest once the previous P V has completed.  (Warps without
    // a row wait as well: their arrivals below must not run ahead.)
    if (j > 0 && !warp_wait(&sb.o_full[w], (j - 1) & 1, abort, p.wait_ns)) {
      ok = false;
      break;
    }
    tc_fence_after_sync();
    if (warp_on) {
#pragma unroll
      for (int c = 0; c < kPfxKeys / 32; ++c) {
        uint32_t q[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) q[k] = pw[16 * c + k];
        tmem_st_32x32b_x16(lane_tmem + p_col + 16 * c, q);
      }
    }
    const bool rescale = live && m_new != m && m != -INFINITY;
    const float f = rescale ? ex2_approx(m - m_new) : 1.0f;
    m = m_new;
    l = l * f + sum;
    // A page id out of range: the merge gives 0 to rows whose sum is no number.
    if (flags & kPfxFaulty) l = __int_as_float(0x7fffffff);
    if (warp_on) {
      if (__any_sync(0xffffffffu, rescale)) {
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          uint32_t v[16];
          tmem_ld_32x32b_x16(lane_tmem + o_col + 16 * c, v);
          tmem_ld_wait(v);
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * f);
          tmem_st_32x32b_x16(lane_tmem + o_col + 16 * c, v);
        }
      }
      tmem_st_wait();
    }
    if (keys % 16 != 0) {
      // The item ends inside a step of 16 keys: its rows of V past the end are
      // whatever the pool or an earlier tile left there, and 0 * NaN would
      // spread.
      if (!warp_wait(&sb.v_full[ent.x & 255], (ent.x >> 8) & 1, abort, p.wait_ns)) {
        ok = false;
        break;
      }
      if (r >= keys && r < (keys + 15) / 16 * 16) {
        const uint32_t row = smem_u32(ring + (NS + (ent.x & 255)) * C::kTileBytes + r * 128);
#pragma unroll 1
        for (int k = 0; k < 8; ++k)
          for (int b = 0; b < C::kBoxes; ++b) st_shared_v4(row + b * 128 * 128 + k * 16, 0u, 0u, 0u, 0u);
        fence_proxy_async_smem();
      }
    }
    tc_fence_before_sync();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sb.p_full[w]);
    if (flags & kPfxLast) {
      if (!warp_wait(&sb.o_full[w], j & 1, abort, p.wait_ns)) {
        ok = false;
        break;
      }
      tc_fence_after_sync();
      const int rows = kind == kPfxOwn ? p.rows : kPfxRows, row = kind == kPfxOwn ? own_r : r;
      float2* ml = kind == kPfxOwn ? p.work.ml[0] : kind == kPfxSingle ? p.work.ml[1] : p.work.ml[2];
      if (row_on) ml[(size_t)ent.w * rows + row] = live ? make_float2(m, l) : make_float2(-INFINITY, 0.0f);
      if (warp_on) {
        float4* O = kind == kPfxOwn ? p.work.O[0] : kind == kPfxSingle ? p.work.O[1] : p.work.O[2];
        float4* out = O + (size_t)ent.w * rows * (D / 4) + row;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_ld_32x32b_x32(lane_tmem + o_col + 32 * c, v);
          tmem_ld_wait(v);
          if (live) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              out[(8 * c + k) * rows] = make_float4(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1]),
                                                    __uint_as_float(v[4 * k + 2]), __uint_as_float(v[4 * k + 3]));
          }
        }
        tc_fence_before_sync();
      }
    }
  }
  tmem_st_wait();
  if (!ok && lane == 0) {
    *reinterpret_cast<volatile int*>(&sb.abort) = 1;
    atomicOr(p.cache.status, kStatusTimeout);
  }
}

// Where the partial results of request and kv head i = req * n_kv_heads + kvh
// lie, as two int4: {n, n_pre, step, kind}, {slot, first row, own slot, 0}.
// The first n_pre are those of the shared prefix, in every step-th slot of its
// kind; the others, of the request's own keys, in consecutive slots.
__device__ __forceinline__ void pfx_sources(const PfxParams& p, const PfxPlan& plan, int i, int4* out) {
  const int kv = p.cache.n_kv_heads;
  const int req = i / kv, kvh = i - req * kv;
  const PfxTotals t = *plan.t;
  const int g = plan.group[req], own_first = plan.cum[req], own_tiles = plan.cum[req + 1] - own_first;
  int n_pre = 0, n_own = 0, step = 1, kind = kPfxSingle, slot = 0, row0 = 0, own_slot = 0;
  if (plan.len[req] > 0) {
    if (g >= 0) {
      const int at = req - plan.start[g], tiles = plan.tiles[g], n_pairs = plan.pairs[g];
      const int tile = at / p.per_tile;
      const bool pair = tile < 2 * n_pairs;
      row0 = (at - tile * p.per_tile) * p.rows;
      const int it = pair ? kvh * n_pairs + tile / 2 : kvh;
      const int x = (pair ? plan.pair_base[g] : plan.single_base[g]) + it * tiles;
      const PfxCuts cuts = pair ? t.pair : t.line;
      const int k0 = pfx_run_of(cuts, x);
      n_pre = pfx_run_of(cuts, x + tiles - 1) - k0 + 1;
      kind = pair ? kPfxPair : kPfxSingle;
      step = pair ? 2 : 1;
      slot = pair ? 2 * (plan.pair_item[g] * kv + it + k0) + (tile & 1) : plan.single_item[g] * kv + it + k0;
    }
    if (own_tiles > 0) {
      const int x = t.single_tiles + own_first * kv + kvh * own_tiles;
      const int k0 = pfx_run_of(t.line, x);
      n_own = pfx_run_of(t.line, x + own_tiles - 1) - k0 + 1;
      own_slot = i + k0;
    }
  }
  out[0] = make_int4(n_pre + n_own, n_pre, step, kind);
  out[1] = make_int4(slot, row0, own_slot, 0);
}

// -------------------------------------------------------------------- kernel
template <int D, bool FP16>
__global__ void __launch_bounds__(PfxCfg<D>::kThreads, 1)
    prefix_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                  const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapQ1,
                  const __grid_constant__ PfxParams p) {
  using C = PfxCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* q_tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = q_tiles + 2 * C::kTileBytes;
  const PfxPlan plan = pfx_plan(reinterpret_cast<int*>(q_tiles + C::kRingBytes), p.batch, p.n_groups);
  __shared__ PfxShared<C::kSlots> sb;
  static_assert(sizeof(sb) <= 1024, "static shared memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    sb.abort = 0;
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(&sb.k_full[i], 1);
      mbar_init(&sb.v_full[i], 1);
      mbar_init(&sb.k_empty[i], 1);
      mbar_init(&sb.v_empty[i], 1);
    }
    for (int w = 0; w < 2; ++w) {
      for (int i = 0; i < kPfxSched; ++i) {
        mbar_init(&sb.sched_full[w][i], 1);
        mbar_init(&sb.sched_empty[w][i], 6);
      }
      mbar_init(&sb.q_full[w], 1);
      mbar_init(&sb.q_free[w], 1);
      mbar_init(&sb.s_full[w], 1);
      mbar_init(&sb.s_free[w], 4);
      mbar_init(&sb.p_full[w], 4);
      mbar_init(&sb.o_full[w], 1);
      mbar_init(&sb.done[w], 1);
    }
    fence_mbar_init();
    tma_prefetch_map(&mapK);
    tma_prefetch_map(&mapV);
    tma_prefetch_map(&mapQ);
    tma_prefetch_map(&mapQ1);
  }
  if (warp == 9) {
    tmem_alloc(&sb.tmem_base, 512);
    tmem_relinquish();
  }
  // Everything above may overlap the previous kernel of the stream.
  griddep_wait();
  tc_fence_before_sync();
  pfx_make_plan(p, plan, blockIdx.x == 0);  // ends with a barrier
  tc_fence_after_sync();
  const uint32_t tmem = sb.tmem_base;
  if (threadIdx.x == 0) griddep_launch_dependents();  // the merge waits for this grid's end

  if (warp < 8) {
    // While the first tiles are on their way: where the merge finds its parts.
    for (int i = blockIdx.x * 256 + threadIdx.x; i < p.batch * p.cache.n_kv_heads; i += gridDim.x * 256)
      pfx_sources(p, plan, i, p.work.sources + 2 * (size_t)i);
    __syncwarp();
    warpgroup_reg_inc<C::kRegsSoftmax>();
    pfx_softmax<D, FP16>(p, plan, warp >> 2, tmem, ring, sb);
  } else {
    warpgroup_reg_dec<C::kRegsOther>();
    if (warp == 8 || warp == 11) {
      pfx_producer<D>(&mapK, &mapV, &mapQ, &mapQ1, p, plan, warp == 11, q_tiles, ring, sb);
    } else if (lane == 0) {
      // The stream that takes the second turn at a pair's tile: stream 1,
      // unless stream 0 had one tile more before.
      const PfxCuts line = plan.t->line;
      int run = (int)blockIdx.x - plan.t->pair.runs;
      if (run < 0) run += gridDim.x;
      const int second = pfx_run_tiles(line, run) == pfx_run_tiles(line, run + gridDim.x);
      if (warp == 9)
        pfx_mma_s<D, FP16>(p, second, tmem, q_tiles, ring, sb);
      else
        pfx_mma_pv<D, FP16>(p, second, tmem, ring, sb);
    }
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    __syncwarp();
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// --------------------------------------------------------------------- merge
// Joins the partial results of one request and kv head; blockIdx.y takes a
// share of the columns.  A thread owns 4 columns of one row; where a block has
// fewer such elements than threads, `parts` threads share an element, each
// taking every parts-th segment.  What bounds it: a chain of three dependent
// loads (the sources, (m, l), O), so blocks are small, many share an SM, and a
// thread has eight loads of O in flight.
constexpr int kMergeThreads = 128;
constexpr int kMergeStats = 1024;  // (m, l) pairs in shared memory at a time

struct PfxMergeShape {
  int log_rows;  // rows of a request rounded up to a power of two
  int cols;      // groups of 4 columns of a block
  int parts;
};

template <int D, bool FP16>
__global__ void __launch_bounds__(kMergeThreads, 12) prefix_merge_kernel(const PfxParams p, const PfxMergeShape sh,
                                                                     uint16_t* O) {
  __shared__ float2 stats[kMergeStats];
  __shared__ float4 sums[kMergeThreads];
  __shared__ float part_l[kMergeThreads];
  griddep_launch_dependents();  // what follows waits for this grid's end
  griddep_wait();
  const int4 s0 = p.work.sources[2 * (size_t)blockIdx.x], s1 = p.work.sources[2 * (size_t)blockIdx.x + 1];
  const int n = s0.x, n_pre = s0.y, pre_step = s0.z, kind = s0.w;
  const int R = p.rows, tid = threadIdx.x;
  const float2* pre_ml = p.work.ml[kind] + (size_t)s1.x * kPfxRows + s1.y;
  const float4* pre_O = p.work.O[kind] + (size_t)s1.x * kPfxRows * (D / 4) + s1.y;
  const float2* own_ml = p.work.ml[kPfxOwn] + (size_t)s1.z * R;
  const float4* own_O = p.work.O[kPfxOwn] + (size_t)s1.z * R * (D / 4);
  const int row_mask = (1 << sh.log_rows) - 1;
  const int row = tid & row_mask;
  const int el = sh.cols << sh.log_rows;         // elements of this block, at most one a thread
  const int part = sh.parts > 1 ? tid / el : 0;
  const int e = tid - part * el;
  const bool on = row < R && part < sh.parts && e < el;
  const int col = blockIdx.y * sh.cols + (e >> sh.log_rows);
  const int chunk = kMergeStats >> sh.log_rows;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float m = -INFINITY, l = 0.0f;
  for (int first = 0; first < n; first += chunk) {
    const int ns = min(chunk, n - first);
    if (first > 0) __syncthreads();
    for (int k = tid; k < ns << sh.log_rows; k += kMergeThreads) {
      const int i = first + (k >> sh.log_rows), rr = k & row_mask;
      if (rr < R)
        stats[k] = i < n_pre ? pre_ml[(size_t)i * pre_step * kPfxRows + rr] : own_ml[(size_t)(i - n_pre) * R + rr];
    }
    __syncthreads();
    if (!on) continue;
    const float m_old = m;
#pragma unroll 4
    for (int i = 0; i < ns; ++i) m = fmaxf(m, stats[(i << sh.log_rows) + row].x);
    if (m == -INFINITY) continue;  // the row saw nothing yet
    const float f = ex2_approx(m_old - m);
    l *= f;
    acc.x *= f;
    acc.y *= f;
    acc.z *= f;
    acc.w *= f;
    // The segments of the prefix in this chunk, then the own ones.  (A segment
    // in which the row saw nothing has m = -inf and O = 0; a row that sees
    // nothing anywhere has no O at all, and l stays 0.)
    auto join = [&](int i0, int i1, const float4* from, size_t step) {
      const float2* st = stats + (i0 << sh.log_rows) + row;
      const int stat_step = sh.parts << sh.log_rows;
#pragma unroll 4
      for (int i = i0; i < i1; i += sh.parts) {
        const float4 v = *from;
        const float u = ex2_approx(st->x - m);
        l += st->y * u;
        acc.x += u * v.x;
        acc.y += u * v.y;
        acc.z += u * v.z;
        acc.w += u * v.w;
        from += step;
        st += stat_step;
      }
    };
    const int pre = min(max(n_pre - first, 0), ns);  // of the chunk
    const size_t pre_seg = (size_t)pre_step * (D / 4) * kPfxRows, own_seg = (size_t)(D / 4) * R;
    join(part, pre, pre_O + (first + part) * pre_seg + col * kPfxRows + row, sh.parts * pre_seg);
    // This thread's next segment after those, counted in steps of `parts`.
    const int i0 = part >= pre ? part : part + (pre - part + sh.parts - 1) / sh.parts * sh.parts;
    join(i0, ns, own_O + (first + i0 - n_pre) * own_seg + col * R + row, sh.parts * own_seg);
  }
  if (sh.parts > 1) {
    sums[tid] = acc;
    part_l[tid] = l;
    __syncthreads();
    if (part == 0) {
      for (int k = 1; k < sh.parts; ++k) {
        const float4 v = sums[tid + k * el];
        acc.x += v.x;
        acc.y += v.y;
        acc.z += v.z;
        acc.w += v.w;
        l += part_l[tid + k * el];
      }
    }
  }
  if (!on || part > 0) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;  // 0 as well where a faulty page made l NaN
  // Row `row` of the request's block of rows of this kv head: Q and O are
  // [batch][n_kv_heads][rows][head_dim].
  uint16_t* out = O + ((size_t)blockIdx.x * R + row) * D + 4 * col;
  *reinterpret_cast<uint2*>(out) =
      make_uint2(pack_16x2<FP16>(acc.x * inv, acc.y * inv), pack_16x2<FP16>(acc.z * inv, acc.w * inv));
}

template <int D, bool FP16>
cudaError_t launch_prefix_instance(const PfxLaunch& L) {
  using C = PfxCfg<D>;
  auto kern = prefix_kernel<D, FP16>;
  const int smem = C::kSmemFixed + pfx_plan_ints(L.p.batch, L.p.n_groups) * 4;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       C::kSmemFixed + C::kMaxPlanBytes);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(L.grid);
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = L.stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if ((e = cudaLaunchKernelEx(&cfg, kern, L.mapK, L.mapV, L.mapQ, L.mapQ1, L.p)) != cudaSuccess) return e;
  // Shares of the columns: at most one element a thread, and more of them (the
  // threads then share elements) while the blocks are few.
  PfxMergeShape sh = {0, D / 4, 1};
  while ((1 << sh.log_rows) < L.p.rows) ++sh.log_rows;
  const long long units = (long long)L.p.batch * L.p.cache.n_kv_heads;
  while (sh.cols > 1 && ((sh.cols << sh.log_rows) > kMergeThreads ||
                         (units * (D / 4 / sh.cols) < 8 * L.grid && (sh.cols << sh.log_rows) > 32)))
    sh.cols = sh.cols % 2 ? 1 : sh.cols / 2;
  sh.parts = kMergeThreads / (sh.cols << sh.log_rows);
  if (sh.parts > 8) sh.parts = 8;
  cfg.gridDim = dim3(L.p.batch * L.p.cache.n_kv_heads, D / 4 / sh.cols);
  cfg.blockDim = dim3(kMergeThreads);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, prefix_merge_kernel<D, FP16>, L.p, sh, reinterpret_cast<uint16_t*>(L.O));
}

template <int D>
cudaError_t launch_prefix_for_dim(bool fp16, const PfxLaunch& L) {
  return fp16 ? launch_prefix_instance<D, true>(L) : launch_prefix_instance<D, false>(L);
}

}  // namespace wise
