// The attention kernel of quant_attn.cuh, one instance per head dimension,
// number of bits and number of rows.
//
// Both products have the cache's side as operand A in tensor memory and the
// query rows (16 to 64 of them) as N:
//   S^T [128 keys x N] = K [keys x D] Q^T,    O^T [D x N] += V^T [D x keys] P^T.
// So a few query rows cost few tensor cycles, and the codes go from shared
// memory through registers right to where the product wants them: a thread
// owns a row of K (a token) or of V^T (a channel), turns 16-byte pieces of
// codes into fp16 pairs and stores those to its lane of tensor memory.
//
// A step is what the softmax takes at once: 256 keys in the narrow instance (up
// to 16 query rows an item), 128 in the wide one (up to 64).  The cache's side
// moves by halves of 128 keys, one row of the product's M each.
//
// Warp roles (768 threads):
//   4 warps      softmax (8 in the wide instance, each 4 for 32 of the rows): S^T
//                from tensor memory in fragments of 8 keys x 8 rows, the mask,
//                running maximum (raised only when a numerator passes 2^15, which
//                the warps vote on), numerators as fp16 to shared memory (P, the B
//                operand of the second product), O's rescaling.  A product takes
//                both operands in one type, and K and V are exact in fp16: P's
//                rounding there, 2^-11, is an eighth of bf16's.  fp16 outputs are
//                off by 2.9e-4 (relative, whole outputs) with it, 2.1e-4 of which
//                is their own rounding; in 32 bits they would take twice the room;
//   4 warps      K: codes to tensor memory;
//   8 or 4       V: the same, scales of 8 tokens at a time (in the narrow instance
//                two teams that take every other half);
//   4 warps      results: O, or a partial result, of segments that have ended,
//                while the softmax goes on with the next;
//   a warp       producer: one bulk copy a page (codes and scales of keys and
//                values lie together), the schedule;
//   a warp       the walk over the segments and their page look-ups, and Q: rows of
//                the next segment to shared memory as fp16, those of bf16 each scaled
//                by a power of two so that its largest is in [2^14, 2^15) (entries are
//                exact down to 2^-31 of it), and how many keys each row sees;
//   two warps    S products and P V products, each issued by one lane.
// All of tensor memory is allocated, so that its first column is 0.
//
// What bounds it.  With 8 bits the memory: 16 x about 4K tokens of 32 kv heads of
// 128 in 103 us, 5.8 TB/s, 0.85 of a copy.  With 4 bits and long rows neither the
// memory nor the issue slots are full (56 and 65 of 100): turning codes into operands
// and the softmax wait for one another's latencies in the rest (32 x 12K tokens of 8
// kv heads: 105 us, 4.4 TB/s, 2300 clk a step).  In the wide instance it is the chain
// S, softmax, P of one step after the other, 1.0 us for 128 keys, which decodes them
// for at most 64 rows (64 requests of 4 rows on a shared 32K prefix: 116 us, where a
// cache of 16 bits takes 70: its items have 256 rows).  With short rows the fetching
// of instructions: 24 warps in a dozen codes of their own keep little of what a
// segment does once in the nearest cache, and code that runs once costs 8 to 10 clk
// an instruction.  So what belongs to a segment is in loops and on warps beside the
// softmax's: with the results on the softmax's warps, the walk on the producer's and
// the copying of Q unrolled, a segment of one step took 8800 clk, now 6400 (5500 items
// of 210 tokens: 169 -> 124 us; of 900 tokens: 228 -> 183 us).  6 to 9 us pass from the
// last step of own keys to the first of a prefix with 64 rows.
//
// Every wait is bounded; one that runs out sets the status word and an abort
// flag, and every role unwinds.
#pragma once

#include <float.h>

#include "attn_common.cuh"
#include "cache_common.cuh"
#include "ptx.cuh"
#include "quant.cuh"
#include "quant_attn.cuh"

namespace wise {

template <int D, int BITS, int NMAX>
struct QaCfg {
  static constexpr int kHalves = NMAX == 16 ? 2 : 1;  // of 128 keys, of a step
  // Warpgroups: softmax, K, V (teams that take the halves in turn), one that writes
  // results, and one for the rest.
  static constexpr int kGroups = NMAX == 16 ? 1 : 2, kKeyTeams = 1, kTeams = NMAX == 16 ? 2 : 1;
  static constexpr int kThreads = 128 * (kGroups + kKeyTeams + kTeams + 2);
  // Halves of K and of V in tensor memory.  V stays until the softmax has been
  // through its step: with 3 buffers one half of a step has to wait for the
  // products of the step before (32 x 12K tokens: 2 us more).
  static constexpr int kKeyBuffers = 2, kValueBuffers = NMAX == 16 ? 4 : 2;
  // Steps whose S and P are held at a time (2 in the wide instance: 64 on a shared
  // 32K prefix 120 -> 128 us), and segments whose O is.
  static constexpr int kDepth = 3, kOuts = NMAX == 16 ? 2 : 1;
  // Columns: K, V, S, O.
  static constexpr uint32_t kTmemK = 0, kTmemV = 64 * kKeyBuffers, kTmemS = kTmemV + 64 * kValueBuffers,
                            kTmemO = kTmemS + kDepth * kHalves * NMAX;
  static_assert(kTmemO + kOuts * NMAX <= 512, "tensor memory");
  static_assert(kKeyTeams <= kTeams, "the end is told to each team of V");
  static constexpr int kBoxes = (D + 63) / 64;
  static constexpr int kBoxBytes = NMAX * 128;
  static constexpr int kQBytes = kBoxes * kBoxBytes;
  static constexpr int kPBytes = 2 * kHalves * kBoxBytes;
  static constexpr int kStageBytes = 128 / 16 * q_block_bytes(BITS, D, 16);  // 128 tokens, whatever the page size
  static constexpr int kMaxPlanBytes = 32 * 1024;
  static constexpr int kSumBytes = 2 * (NMAX / 8) * 128 * 8;  // of two steps, a pair of rows' sums for each thread
  static constexpr int kFixed = 2 * kQBytes + kDepth * kPBytes + kSumBytes;
  static constexpr int kRoom = (217 * 1024 - 1024 - kMaxPlanBytes - kFixed) / kStageBytes;
  // A multiple of the V teams.  A wait knows the parity of a stage's phase alone,
  // so whoever waits for a load must have seen the stage's load before it, and a
  // team sees its own halves only (loads may end out of order).
  static constexpr int kStages = (kRoom < 8 ? kRoom : 8) / kTeams * kTeams;
  static constexpr int kPlanAt = kFixed + kStages * kStageBytes;
  static constexpr int kSmem = kPlanAt + kMaxPlanBytes + 1024;
  static_assert(kStages >= 2 && kStageBytes % 128 == 0 && kValueBuffers % kTeams == 0, "rings");
};

constexpr int kQaSched = 16;
constexpr int kQaFirst = 1, kQaLast = 2, kQaEnd = 4, kQaFaulty = 8;
constexpr int kQaOwn = 0, kQaPrefix = 1;

// Segment entry, two int4: {rows | kind << 8 (0: the end), position of the first
// key, of the last one + 1, request}, {kv head, first row of the request,
// workspace slot or -1 (O itself), cache row}, and its first 32 pages, one a lane.
// Entry k % 16 is written again for segment k + 16, after the queries of segment
// k + 14 have found a buffer and so after segment k's results.
//
// Schedule entry of a step: {flags | rows << 8 | kind << 16 | keys << 20, position
// of the first key}.  The K and V warps go by halves and need no more than
// half_keys, which comes with the stage.  Entry t % 16 is written again for step
// t + 16, whose first stage (of at most 8) the V warps have given back: they are
// at most 4 halves ahead of the products of P, and so of the softmax, which is
// past step t then.
__device__ __forceinline__ int qa_rows(int info) { return (info >> 8) & 255; }
__device__ __forceinline__ int qa_kind(int info) { return (info >> 16) & 1; }
__device__ __forceinline__ int qa_keys_of(int info) { return info >> 20; }

template <int NS, int NK, int NV, int NT, int NG, int ND>
struct QaShared {
  uint64_t full[NS], empty[NS];  // empty: 8 warps
  uint64_t sched_full[kQaSched], seg_full[kQaSched];
  uint64_t k_ready[NK], k_free[NK];  // 4 warps; products
  uint64_t v_ready[NV], v_free[NV];
  uint64_t p_ready[ND];              // softmax warps
  uint64_t s_full[ND], s_free[ND];   // products; softmax warps
  uint64_t pv_done[ND];
  uint64_t o_full[2], o_free[2];     // a segment's products; 4 warps that have read O
  uint64_t end_ready[2];             // softmax warps: what ends a segment is written
  uint64_t q_ready[2], q_free[2];  // q_free: the products and the softmax warps
  uint64_t done[2];
  int2 sched[kQaSched];
  int4 segs[kQaSched][2];
  int pages[kQaSched][32];
  alignas(16) int lim[2][kQaRows];  // keys that a row sees, 0 for none
  int min_lim[2];            // the least of those that see any
  int q_from[kQaRows];       // where a row comes from, -1 for a row of 0
  alignas(16) float q_scale[2][kQaRows];  // a row's logits in base-2 units = S * q_scale
  alignas(16) float warp_max[2][4][kQaRows];
  alignas(16) float shift[2][kQaRows];  // added to a row's logits: 7 minus the reference, 0 where nothing is seen
  alignas(16) float top[2][kQaRows];    // the reference less 7, -inf where nothing is seen
  alignas(16) float factor[kQaRows];    // of O and the sums where the references have moved
  // Of a segment that ends: its flags and its rows' sums by warp.
  int last[2];
  alignas(16) float sums[2][4][kQaRows];
  alignas(16) int4 value_scales[4 * NT][32];  // a warp's two groups x 128 tokens as fp16
  int half_keys[NS];  // keys of the half in a stage, 0 at the end
  uint32_t tmem_base;
  int abort, failed[NG];  // failed: a wait of one of the group's warps has run out
};

// ---------------------------------------------------------------------- plan
// All threads; `plan` in shared memory.
__device__ inline void qa_make_plan(const QaParams& p, const QaPlan& plan, bool report) {
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
  const bool grouped = !__syncthreads_or(bad_groups) && p.per_tile > 0;
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
    if (lane == 0) {
      const int tiles = (shared + p.keys - 1) / p.keys;
      const int row_tiles = tiles > 0 ? (e - a + p.per_tile - 1) / p.per_tile : 0;
      plan.tiles[g] = tiles;
      plan.lead[g] = lead;
      plan.row_tiles[g] = row_tiles;
      plan.base[g] = row_tiles * tiles * c.n_kv_heads;
      plan.item[g] = row_tiles;
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
  // Prefix sums, a warp each: the groups' tiles and items, the requests' own tiles.
  if (warp < 3) {
    int* list = warp == 0 ? plan.base : warp == 1 ? plan.item : plan.cum;
    const int n = warp < 2 ? p.n_groups : p.batch;
    int before = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += 128) {
      const int first = i0 + 4 * lane;
      int x[4], sum = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = 0;
        if (first + k < n)
          x[k] = warp < 2 ? list[first + k]
                          : max(0, plan.len[first + k] - plan.lo[first + k] + p.keys - 1) / p.keys;
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
  if (tid < 2) {
    const PfxCuts cuts =
        pfx_cuts(tid == 0 ? plan.cum[p.batch] * c.n_kv_heads * p.chunks : plan.base[p.n_groups], gridDim.x);
    (tid == 0 ? plan.t->own : plan.t->pre) = cuts;
  }
  __syncthreads();
}

__device__ __forceinline__ int qa_find(const int* base, int n, int x) {
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

struct QaSeg {
  int kind, req, kvh;
  int row0, rows;  // first row of the request (own), rows
  int seq, pos, end;  // cache row, positions of the first key and of the last one + 1
  int slot;        // workspace slot, -1 for O itself
  int left;        // tiles
};

// Walks a CTA's segments: its run of own items, then its run of prefix items.
// Runs of own items start at the CTA after the last one with prefix items, so
// that small problems spread out.  The first item of a run is found by a search
// and divisions, the others by steps: short items need a segment every few
// microseconds.
struct QaWalk {
  int kind = -1, run, x = 0, x_end = 0;
  int t;           // of the next item: its first tile
  int req, kvh, row0;  // own: the item
  int g, it, tile;     // prefix: the group, the item in it, and the item among those of its kv head
  __device__ __forceinline__ void begin(const QaParams& p, const QaPlan& plan, int k) {
    kind = k;
    const PfxCuts c = k == kQaOwn ? plan.t->own : plan.t->pre;
    run = blockIdx.x;
    if (k == kQaOwn) {
      run -= plan.t->pre.runs;
      if (run < 0) run += gridDim.x;
    }
    x = x_end = 0;
    if (run >= c.runs) return;
    x = pfx_cut(c, run);
    x_end = pfx_cut(c, run + 1);
    if (k == kQaOwn) {
      const int per = p.cache.n_kv_heads * p.chunks;
      req = qa_find(plan.cum, p.batch, x / per);  // cum[r] * per <= x < cum[r + 1] * per
      const int tiles = plan.cum[req + 1] - plan.cum[req], z = x - plan.cum[req] * per, unit = z / tiles;
      t = z - unit * tiles;
      kvh = unit / p.chunks;
      row0 = (unit - kvh * p.chunks) * kQaRows;
    } else {
      g = qa_find(plan.base, p.n_groups, x);
      const int tiles = plan.tiles[g], y = x - plan.base[g], n = plan.row_tiles[g];
      it = y / tiles;
      t = y - it * tiles;
      // kv head outermost: the items of one kv head read the same keys at about the same time.
      kvh = it / n;
      tile = it - kvh * n;
    }
  }
  __device__ __forceinline__ bool next(const QaParams& p, const QaPlan& plan, QaSeg& s) {
    while (x == x_end) {
      if (kind == kQaPrefix) return false;
      begin(p, plan, kind + 1);
    }
    const int kv = p.cache.n_kv_heads;
    int tiles;
    s.kind = kind;
    s.kvh = kvh;
    if (kind == kQaOwn) {
      while (plan.cum[req + 1] == plan.cum[req]) ++req;
      tiles = plan.cum[req + 1] - plan.cum[req];
      s.req = req;
      s.row0 = row0;
      s.rows = min(p.rows - row0, kQaRows);
      s.slot = (req * kv + kvh) * p.chunks + row0 / kQaRows + run;
      s.seq = plan.slot[req];
      s.end = plan.len[req];
      s.pos = plan.lo[req] + t * p.keys;
      if (t == 0 && tiles <= x_end - x && plan.group[req] < 0) s.slot = -1;
      row0 += kQaRows;
      if (row0 >= p.rows) {
        row0 = 0;
        if (++kvh == kv) {
          kvh = 0;
          ++req;
        }
      }
    } else {
      while (plan.base[g + 1] == plan.base[g]) ++g;
      tiles = plan.tiles[g];
      s.req = plan.start[g] + tile * p.per_tile;
      s.row0 = 0;
      s.rows = min(p.per_tile, plan.start[g + 1] - s.req) * p.rows;
      s.slot = plan.item[g] * kv + it + run;
      const int lead = plan.lead[g];
      s.seq = plan.slot[lead];
      s.end = plan.lo[lead];
      s.pos = t * p.keys;
      ++it;
      if (++tile == plan.row_tiles[g]) {
        tile = 0;
        if (++kvh == kv) {
          kvh = it = 0;
          ++g;
        }
      }
    }
    s.left = min(tiles - t, x_end - x);
    x += s.left;
    t = 0;
    return true;
  }
};

// Waits.  One that runs out tells everybody: the abort flag ends the others.
struct QaWait {
  int* abort;
  int* status;
  unsigned long long limit;
};
static __device__ __noinline__ void qa_give_up(int* abort, int* status) {
  *reinterpret_cast<volatile int*>(abort) = 1;
  atomicOr(status, kStatusTimeout);
}
// After a first try, which the hardware holds for some microseconds.
static __device__ __noinline__ bool qa_wait_long(uint64_t* bar, uint32_t parity, volatile int* abort, int* status,
                                                 unsigned long long limit) {
  const uint64_t t0 = global_timer_ns() - 1000;
  for (;;) {
    if (__any_sync(0xffffffffu, *abort != 0 || global_timer_ns() - t0 > limit)) {
      if ((threadIdx.x & 31) == 0) qa_give_up(const_cast<int*>(abort), status);
      return false;
    }
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  }
}
// All lanes of a warp.
__device__ __forceinline__ bool qa_wait(uint64_t* bar, uint32_t parity, const QaWait& w) {
  if (__builtin_expect(__all_sync(0xffffffffu, mbar_try_wait(bar, parity)), 1)) return true;
  return qa_wait_long(bar, parity, w.abort, w.status, w.limit);
}

// Two phases, with one latency where both are complete.
__device__ __forceinline__ bool qa_wait_both(uint64_t* a, uint32_t parity_a, uint64_t* b, uint32_t parity_b,
                                             const QaWait& w) {
  const bool first = mbar_test_wait(a, parity_a), second = mbar_test_wait(b, parity_b);
  if (__builtin_expect(__all_sync(0xffffffffu, first && second), 1)) return true;
  return qa_wait(a, parity_a, w) && qa_wait(b, parity_b, w);
}

// A place in a ring of N, and how often the ring has been passed.
template <int N>
struct QaRing {
  int at = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int k = 1) {
    at += k;
    if (at >= N) {
      at -= N;
      phase ^= 1;
    }
  }
};

// One lane of a warp arrives (without a branch around it).
__device__ __forceinline__ void qa_arrive(uint64_t* bar, int lane) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.eq.s32 p, %1, 0;\n\t"
      "@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(smem_u32(bar)),
      "r"(lane)
      : "memory");
}

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

#define QA_SHARED QaShared<QaCfg<D, BITS, NMAX>::kStages, QaCfg<D, BITS, NMAX>::kKeyBuffers, \
                                QaCfg<D, BITS, NMAX>::kValueBuffers, QaCfg<D, BITS, NMAX>::kTeams, \
                                QaCfg<D, BITS, NMAX>::kGroups, QaCfg<D, BITS, NMAX>::kDepth>

// ------------------------------------------------------------------ producer
template <int D, int BITS, int NMAX>
__device__ void qa_producer(const QaParams& p, uint8_t* ring, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  constexpr int NS = C::kStages, kKeys = 128 * C::kHalves;
  const CacheView& c = p.cache;
  const int lane = threadIdx.x & 31;
  const int block = c.head_bytes, half_pages = 128 >> c.page_shift;
  QaRing<NS> st;
  int n = 0, t = 0, bad = 0;
  bool ok = true;
  for (int k = 0;; ++k) {
    if (!(ok = qa_wait(&sb.seg_full[k % kQaSched], (k / kQaSched) & 1, wt))) break;
    const int4 a = sb.segs[k % kQaSched][0], e = sb.segs[k % kQaSched][1];
    if (a.x == 0) break;
    int info = a.x << 8 | kQaFirst, at = 0;  // (rows << 8 | kind << 16); the next half's first lane
    int page = sb.pages[k % kQaSched][lane];
    uint32_t valid = __ballot_sync(0xffffffffu, valid_page(c, page));
    const int* table = c.table + (size_t)e.w * c.max_pages;
    const uint8_t* from = p.plane + (size_t)e.x * block;
#pragma unroll 1
    for (int pos = a.y; pos < a.z; pos += kKeys, info &= ~kQaFirst) {
      if (at == 32) {  // (steps have 1 to 16 pages)
        const int mine = (pos >> c.page_shift) + lane;
        page = mine << c.page_shift < a.z ? __ldg(table + mine) : -1;
        valid = __ballot_sync(0xffffffffu, valid_page(c, page));
        at = 0;
      }
      const int keys = min(kKeys, a.z - pos);
      const uint32_t step = (1u << ((keys + c.page - 1) >> c.page_shift)) - 1u;
      if (step & ~(valid >> at)) {
        info |= kQaFaulty;
        bad = 1;
      }
      if (pos + kKeys >= a.z) info |= kQaLast;
      bool told = false;
#pragma unroll 1
      for (int h = 0; h < keys; h += 128, at += half_pages) {
        if (n >= NS && !(ok = qa_wait(&sb.empty[st.at], st.phase ^ 1, wt))) break;
        if (lane == 0) {
          if (!told) {
            sb.sched[t % kQaSched] = make_int2(info | keys << 20, pos);
            mbar_arrive(&sb.sched_full[t % kQaSched]);
          }
          sb.half_keys[st.at] = min(128, keys - h);
          mbar_arrive_expect_tx(&sb.full[st.at], __popc(valid >> at & ((1u << half_pages) - 1u)) * block);
        }
        __syncwarp();
        const int mine = lane - at;
        if (mine >= 0 && mine < half_pages && (valid >> lane & 1u))
          bulk_load(ring + st.at * C::kStageBytes + mine * block, from + (size_t)page * c.page_bytes, block,
                    &sb.full[st.at]);
        told = true;
        st.next();
        ++n;
      }
      if (!ok) break;
      ++t;
    }
    if (!ok) break;
  }
  // The end, for each of the teams.
#pragma unroll 1
  for (int k = 0; ok && k < C::kTeams; ++k) {
    if (n >= NS && !(ok = qa_wait(&sb.empty[st.at], st.phase ^ 1, wt))) break;
    if (lane == 0) {
      if (k == 0) {
        sb.sched[t % kQaSched] = make_int2(kQaEnd, 0);
        mbar_arrive(&sb.sched_full[t % kQaSched]);
      }
      sb.half_keys[st.at] = 0;
      mbar_arrive(&sb.full[st.at]);
    }
    st.next();
    ++n;
  }
  if (bad && lane == 0) atomicOr(c.status, kStatusBadCache);
  if (lane == 0) {
    // Copies already issued land before the CTA's shared memory is released,
    // whoever may have given up: the last phase of each stage is waited for, that
    // of an end too, as a wait for the phase before it would run out.
    int never = 0;
    for (int k = max(0, n - NS); k < n; ++k) mbar_wait(&sb.full[k % NS], (k / NS) & 1, &never);
  }
  __syncwarp();
}

// ------------------------------------------------------------------------- Q
__device__ __forceinline__ uint32_t qa_pack_half(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int D, int BITS, int NMAX>
__device__ void qa_queries(const QaParams& p, const QaPlan& plan, uint8_t* q_tiles, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  constexpr int kPieces = D / 8;  // of 16 bytes, of a row
  const int lane = threadIdx.x & 31;
  const CacheView& c = p.cache;
  QaWalk walk;
  QaSeg seg = {};
  int page = -1;
  auto next = [&]() {  // the next segment and its first pages
    seg.rows = 0;
    page = -1;
    if (!walk.next(p, plan, seg)) return;
    seg.end = min(seg.end, seg.pos + seg.left * p.keys);
    const int mine = (seg.pos >> c.page_shift) + lane;
    if (mine << c.page_shift < seg.end) page = __ldg(c.table + (size_t)seg.seq * c.max_pages + mine);
  };
  auto tell = [&](int k) {
    sb.pages[k % kQaSched][lane] = page;
    if (lane == 0) {
      sb.segs[k % kQaSched][0] = make_int4(seg.rows | (seg.rows ? seg.kind << 8 : 0), seg.pos, seg.end, seg.req);
      sb.segs[k % kQaSched][1] = make_int4(seg.kvh, seg.row0, seg.slot, seg.seq);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sb.seg_full[k % kQaSched]);
  };
  next();
  tell(0);
#pragma unroll 1
  for (int k = 0;; ++k) {
    const int kvh = seg.kvh, row0 = seg.row0, rows = seg.rows, kind = seg.kind, req = seg.req, end = seg.end;
    if (rows == 0) break;
    const int buf = k & 1;
    if (k >= 2 && !qa_wait(&sb.q_free[buf], ((k >> 1) - 1) & 1, wt)) break;
    // Loops are left as loops: a segment's code is not in the nearest cache when
    // it begins, and straight code costs its fetch.
    const int all = (rows + 15) & ~15;
    int least = INT_MAX;
#pragma unroll 1
    for (int n = lane; n < all; n += 32) {
      int lim = 0, r = 0;
      if (n < rows) {
        if (kind != kQaOwn) r = n * p.rows_inv >> 16;  // n / p.rows
        const int row = row0 + n - r * p.rows, i = row - (row * p.q_len_inv >> 16) * p.q_len, from = req + r;
        if (i < plan.add[from]) lim = max(min(plan.len[from] - plan.add[from] + i + 1, end), 0);
        if (lim > 0) least = min(least, lim);
      }
      // 0 behind the rows too: what a step's empty half holds from before must
      // not look like a numerator there.
      sb.lim[buf][n] = lim;
      sb.q_scale[buf][n] = fmaxf(p.scale_log2, FLT_MIN);
      sb.q_from[n] = lim > 0 ? n + r * (p.cache.n_kv_heads - 1) * p.rows : -1;  // in rows
    }
    least = __reduce_min_sync(0xffffffffu, least);
    if (lane == 0) sb.min_lim[buf] = least;
    __syncwarp();
    // Rows of one request are contiguous: Q is [batch][n_kv_heads][rows][D].  A
    // row takes kPieces lanes.  Rows up to the product's N, and those that see
    // nothing (which may hold anything), are 0.
    constexpr int kAtOnce = 32 / kPieces;
    const int sub = lane / kPieces, piece = lane - sub * kPieces;
    const uint8_t* Q = reinterpret_cast<const uint8_t*>(p.Q) +
                       (((size_t)req * p.cache.n_kv_heads + kvh) * p.rows + row0) * (D * 2) + 16 * piece;
    uint8_t* tile = q_tiles + buf * C::kQBytes + (piece >> 3) * C::kBoxBytes;
#pragma unroll 1
    for (int n = sub; n < all && sub < kAtOnce; n += kAtOnce) {
      const int from = sb.q_from[n];
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                       smem_u32(tile + n * 128 + (((piece & 7) ^ (n & 7)) << 4))),
                   "l"(Q + (size_t)max(from, 0) * (D * 2)), "r"(from < 0 ? 0 : 16)
                   : "memory");
    }
    next();  // the next segment and its pages, while these are on their way
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!p.fp16) {
#pragma unroll 1
      for (int n = sub; n < all + sub; n += kAtOnce) {
        const bool on = sub < kAtOnce && n < all;
        uint4* const at = reinterpret_cast<uint4*>(tile + min(n, all - 1) * 128 + (((piece & 7) ^ (n & 7)) << 4));
        uint4 v = make_uint4(0, 0, 0, 0);
        if (on) v = *at;
        // The row's largest size has exponent field E; times 2^(141 - E) it lies in [2^14, 2^15).
        uint32_t top = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu),
                                __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
        top = max(top & 0xFFFFu, top >> 16);
        if constexpr (kPieces == 12) {
          // 12 lanes: those of the other row keep their own maximum.
          const uint32_t mine = __reduce_max_sync(0xffffffffu, sub == 0 ? top : 0u);
          const uint32_t other = __reduce_max_sync(0xffffffffu, sub == 1 ? top : 0u);
          top = sub == 0 ? mine : other;
        } else {
#pragma unroll
          for (int x = 1; x < kPieces; x <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, x));
        }
        const int shift = top == 0 ? 0 : min(141 - (int)(top >> 7), 126);
        const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = qa_pack_half(__uint_as_float(w[j] << 16) * up, __uint_as_float(w[j] & 0xFFFF0000u) * up);
        if (on) {
          *at = v;
          if (piece == 0)
            sb.q_scale[buf][n] = fmaxf(p.scale_log2 * __uint_as_float((uint32_t)(127 - shift) << 23), FLT_MIN);
        }
      }
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sb.q_ready[buf]);
    tell(k + 1);
  }
  __syncwarp();
}

// ------------------------------------------------------------------ products
// A warp each walks the steps and one lane issues, so that addresses and
// descriptors stay in uniform registers, where the instruction wants them.
__device__ __forceinline__ bool elect_one() {
  uint32_t on;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(on));
  return on != 0;
}

// fp16 operands, fp32 sums; N as in the entry, rounded up to 16 (N / 8 at bit 17).
__device__ __forceinline__ uint32_t qa_idesc(int info) {
  constexpr uint32_t base = idesc_bf16_f32(128, 0, false, false) & ~((1u << 7) | (1u << 10));
  return base | (uint32_t)((qa_rows(info) + 15) >> 4) << 18;
}

// All products of this warp end before tensor memory is given back.
__device__ __forceinline__ void qa_products_done(uint64_t* done) {
  if (elect_one()) {
    int never = 0;
    umma_commit(done);
    mbar_wait(done, 0, &never);
  }
  __syncwarp();
}

template <int D, int BITS, int NMAX>
__device__ void qa_products_s(const QaParams& p, uint8_t* q_tiles, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  const uint64_t desc = smem_desc_sw128(0, 16, 1024);
  const uint32_t hi = (uint32_t)(desc >> 32), q_lo = (uint32_t)desc + (smem_u32(q_tiles) >> 4);
  QaRing<C::kKeyBuffers> kb;
  QaRing<C::kDepth> r;
  int seg = -1;
#pragma unroll 1
  for (int t = 0;; ++t, r.next()) {
    if (!qa_wait(&sb.sched_full[t % kQaSched], (t / kQaSched) & 1, wt)) break;
    const int info = __shfl_sync(0xffffffffu, sb.sched[t % kQaSched].x, 0);
    const int b = r.at;
    // (The end too waits for the softmax to have seen the step that had this buffer.)
    if (t >= C::kDepth && !qa_wait(&sb.s_free[b], r.phase ^ 1, wt)) break;
    if (info & kQaEnd) {
      if (elect_one()) {
        mbar_arrive(&sb.s_full[b]);
        mbar_arrive(&sb.s_full[b]);
      }
      __syncwarp();
      break;
    }
    if (info & kQaFirst) {
      ++seg;
      if (!qa_wait(&sb.q_ready[seg & 1], (seg >> 1) & 1, wt)) break;
    }
    const uint32_t idesc = qa_idesc(info), q0 = q_lo + (seg & 1) * (C::kQBytes >> 4);
    bool ok = true;
#pragma unroll 1
    for (int h = 0; 128 * h < qa_keys_of(info); ++h) {
      if (!(ok = qa_wait(&sb.k_ready[kb.at], kb.phase, wt))) break;
      tc_fence_after_sync();
      const uint32_t s_at = C::kTmemS + (b * C::kHalves + h) * NMAX, k_at = C::kTmemK + 64 * kb.at;
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          umma_ts_split(s_at, k_at + 8 * kk, q0 + (((kk >> 2) * C::kBoxBytes + (kk & 3) * 32) >> 4), hi, idesc, kk > 0);
        umma_commit(&sb.k_free[kb.at]);
        if (128 * (h + 1) >= qa_keys_of(info)) {
          umma_commit(&sb.s_full[b]);
          if (info & kQaLast) umma_commit(&sb.q_free[seg & 1]);
        }
      }
      __syncwarp();
      kb.next();
    }
    // The softmax also learns here what this warp knows: the schedule, the
    // queries, and that P's buffer has been read (a wait less on its own way).
    if (!ok || (t >= C::kDepth && !qa_wait(&sb.pv_done[b], r.phase ^ 1, wt))) break;
    if (elect_one()) mbar_arrive(&sb.s_full[b]);
    __syncwarp();
  }
  qa_products_done(&sb.done[0]);
}

template <int D, int BITS, int NMAX>
__device__ void qa_products_pv(const QaParams& p, uint8_t* p_tiles, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  const uint64_t desc = smem_desc_sw128(0, 16, 1024);
  const uint32_t hi = (uint32_t)(desc >> 32), p_lo = (uint32_t)desc + (smem_u32(p_tiles) >> 4);
  QaRing<C::kValueBuffers> vb;
  QaRing<C::kDepth> r;
  int seg = -1;
#pragma unroll 1
  for (int t = 0;; ++t, r.next()) {
    if (!qa_wait(&sb.sched_full[t % kQaSched], (t / kQaSched) & 1, wt)) break;
    const int info = __shfl_sync(0xffffffffu, sb.sched[t % kQaSched].x, 0);
    if (info & kQaEnd) break;
    const int b = r.at;
    if (!qa_wait(&sb.p_ready[b], r.phase, wt)) break;
    if (info & kQaFirst) {
      ++seg;
      if (const int old = seg - C::kOuts; old >= 0 && !qa_wait(&sb.o_free[old & 1], (old >> 1) & 1, wt)) break;
    }
    const uint32_t idesc = qa_idesc(info), o_at = C::kTmemO + seg % C::kOuts * NMAX;
    bool ok = true;
#pragma unroll 1
    for (int h = 0; 128 * h < qa_keys_of(info); ++h) {
      if (!(ok = qa_wait(&sb.v_ready[vb.at], vb.phase, wt))) break;
      tc_fence_after_sync();
      const uint32_t p0 = p_lo + ((b * C::kPBytes + 2 * h * C::kBoxBytes) >> 4), v_at = C::kTmemV + 64 * vb.at;
      const uint32_t more = h > 0 || !(info & kQaFirst);
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          umma_ts_split(o_at, v_at + 8 * kk, p0 + (((kk >> 2) * C::kBoxBytes + (kk & 3) * 32) >> 4), hi, idesc,
                        kk > 0 ? 1 : more);
        umma_commit(&sb.v_free[vb.at]);
        if (128 * (h + 1) >= qa_keys_of(info)) {
          umma_commit(&sb.pv_done[b]);
          if (info & kQaLast) umma_commit(&sb.o_full[seg & 1]);
        }
      }
      __syncwarp();
      vb.next();
    }
    if (!ok) break;
  }
  qa_products_done(&sb.done[1]);
}

// ------------------------------------------------------------ K and V to TMEM
// Word of codes -> fp16 pairs.
template <int BITS>
struct QaDecode;
template <>
struct QaDecode<4> {
  static constexpr int kPairs = 4;  // of a word
  __device__ static __forceinline__ void pairs(uint32_t w, uint32_t (&h)[4]) { q_decode4(w, h); }
};
template <>
struct QaDecode<8> {
  static constexpr int kPairs = 2;
  __device__ static __forceinline__ void pairs(uint32_t w, uint32_t (&h)[2]) { q_decode8(w, h); }
};

// A thread owns a token: 32 of its values (two groups) at a time.
template <int D, int BITS, int NMAX>
__device__ void qa_keys(const QaParams& p, int team, uint8_t* ring, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  const CacheView& c = p.cache;
  const int lane = threadIdx.x & 31, quarter = (threadIdx.x >> 5) & 3;
  const int token = 32 * quarter + lane, off = token & (c.page - 1);
  const int block_at = (token >> c.page_shift) * c.head_bytes;
  const uint8_t* data_at = ring + block_at + off * 16;
  const uint8_t* scales_at = ring + block_at + q_key_scales_at(BITS, D, c.page) + off * q_key_scale_bytes(D);
  const int step = c.page * 16;  // from 16 bytes of a token to the next 16
  const uint32_t to = ((uint32_t)(32 * quarter) << 16) + C::kTmemK;
  QaRing<C::kStages> st;
  QaRing<C::kKeyBuffers> kb;
  st.next(team);
  kb.next(team);
#pragma unroll 1
  for (int u = team;; u += C::kKeyTeams) {  // halves
    // (A buffer that has not been used yet counts as free: its phase before the first.)
    if (!qa_wait_both(&sb.full[st.at], st.phase, &sb.k_free[kb.at], kb.phase ^ 1, wt)) return;
    const int keys = sb.half_keys[st.at];
    if (keys == 0) return;
    tc_fence_after_sync();
    const uint8_t* data = data_at + st.at * C::kStageBytes;
    const uint8_t* scales = scales_at + st.at * C::kStageBytes;
    // kTogether pieces of 32 values at a time: all of them in the narrow instance
    // of 4 bits, whose K warps then wait for shared memory once.
    constexpr int kTogether = BITS == 4 && NMAX == 16 ? D / 32 : 1;
#pragma unroll 1
    for (int d0 = 0; d0 < D / 32; d0 += kTogether) {
      uint32_t w[kTogether][BITS];
      uint16_t both[kTogether];
#pragma unroll
      for (int d = 0; d < kTogether; ++d) {
        both[d] = *reinterpret_cast<const uint16_t*>(scales + 2 * (d0 + d));
#pragma unroll
        for (int k = 0; k < BITS; k += 4) {
          *reinterpret_cast<uint4*>(w[d] + k) = *reinterpret_cast<const uint4*>(data);
          data += step;
        }
      }
#pragma unroll
      for (int d = 0; d < kTogether; ++d) {
        const uint32_t s0 = (both[d] & 255) * 0x00800080u, s1 = (uint32_t)(both[d] >> 8) * 0x00800080u;
        uint32_t r[16];
#pragma unroll
        for (int k = 0; k < BITS; ++k) {
          constexpr int kPairs = QaDecode<BITS>::kPairs;
          uint32_t x[kPairs];
          QaDecode<BITS>::pairs(w[d][k], x);
#pragma unroll
          for (int j = 0; j < kPairs; ++j) r[k * kPairs + j] = q_mul2(x[j], k < BITS / 2 ? s0 : s1);
        }
        tmem_st_32x32b_x16(to + 64 * kb.at + 16 * (d0 + d), r);
      }
    }
    __syncwarp();
    qa_arrive(&sb.empty[st.at], lane);
    tmem_st_wait();
    tc_fence_before_sync();
    __syncwarp();
    qa_arrive(&sb.k_ready[kb.at], lane);
    st.next(C::kKeyTeams);
    kb.next(C::kKeyTeams);
  }
}

// A thread owns a channel: 32 tokens at a time.
template <int D, int BITS, int NMAX>
__device__ void qa_values(const QaParams& p, int team, uint8_t* ring, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  const CacheView& c = p.cache;
  const int lane = threadIdx.x & 31, quarter = (threadIdx.x >> 5) & 3;
  const bool on = 32 * quarter < D;
  const int T = q_value_tokens(BITS, c.page), piece = T * BITS / 8;  // tokens and bytes of a piece
  const int values_at = q_values_at(BITS, D, c.page) + (32 * quarter + lane) * piece;
  // From 32 tokens to the next 32 (in turn, as pages of 64 have two of them), and
  // from their first 16 to the others where those lie apart.
  const int inside = 32 / T * D * piece;
  const int even = c.page == 16 ? 2 * c.head_bytes : c.page == 32 ? c.head_bytes : inside;
  const int odd = c.page == 64 ? c.head_bytes - inside : even;
  const int apart = c.page == 16 ? c.head_bytes : D * piece;
  // Scales: this lane turns those of 8 tokens of one of the warp's two groups into fp16.
  const int stoken = 8 * (lane & 15);
  const int scales_at = (stoken >> c.page_shift) * c.head_bytes + q_value_scales_at(BITS, D, c.page) +
                        (2 * quarter + (lane >> 4)) * c.page + (stoken & (c.page - 1));
  const uint32_t to = ((uint32_t)(32 * quarter) << 16) + C::kTmemV;
  QaRing<C::kStages> st;
  QaRing<C::kValueBuffers> vb;
  st.next(team);
  vb.next(team);
#pragma unroll 1
  for (int u = team;; u += C::kTeams) {  // halves
    // (A buffer that has not been used yet counts as free: its phase before the first.)
    if (!qa_wait_both(&sb.full[st.at], st.phase, &sb.v_free[vb.at], vb.phase ^ 1, wt)) return;
    const int keys = sb.half_keys[st.at];
    if (keys == 0) return;
    tc_fence_after_sync();
    if (on) {
      const uint8_t* stage = ring + st.at * C::kStageBytes;
      const uint2 bytes = *reinterpret_cast<const uint2*>(stage + scales_at);
      uint32_t s[4];
      s[0] = __byte_perm(bytes.x, 0, 0x1404) >> 1;  // bytes 0 and 1, each shifted by 7 in its half
      s[1] = __byte_perm(bytes.x, 0, 0x3424) >> 1;
      s[2] = __byte_perm(bytes.y, 0, 0x1404) >> 1;
      s[3] = __byte_perm(bytes.y, 0, 0x3424) >> 1;
      if (__builtin_expect(keys < 128, 0)) {  // tokens past the end count 0 whatever is stored there
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (stoken + 2 * k >= keys) s[k] = 0;
          if (stoken + 2 * k + 1 >= keys) s[k] &= 0xFFFFu;
        }
      }
      __syncwarp();  // the scales of the half before have been read
      sb.value_scales[4 * team + quarter][lane] = *reinterpret_cast<const int4*>(s);
      __syncwarp();
      const int4* scales = &sb.value_scales[4 * team + quarter][lane & 16];
      const uint8_t* from = stage + values_at;
#pragma unroll 1
      for (int token = 0; token < 128; token += 32) {
        uint32_t w[BITS], r[16];
        if constexpr (BITS == 8) {
          *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(from);
          *reinterpret_cast<uint4*>(w + 4) = *reinterpret_cast<const uint4*>(from + apart);
        } else if (T == 32) {
          *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(from);
        } else {
          *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(from);
          *reinterpret_cast<uint2*>(w + 2) = *reinterpret_cast<const uint2*>(from + apart);
        }
        from += token & 32 ? odd : even;
        if (BITS == 8 && __builtin_expect(token + 32 > keys, 0)) {  // a code may be NaN there
#pragma unroll
          for (int k = 0; k < BITS; ++k) {
            const int n = min(max(keys - token - 4 * k, 0), 4);
            w[k] = n == 4 ? w[k] : w[k] & ((1u << 8 * n) - 1u);
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // 8 tokens
          const int4 f = scales[token / 8 + q];
          const uint32_t fs[4] = {(uint32_t)f.x, (uint32_t)f.y, (uint32_t)f.z, (uint32_t)f.w};
          constexpr int kPairs = QaDecode<BITS>::kPairs;
#pragma unroll
          for (int k = 0; k < BITS / 4; ++k) {
            uint32_t x[kPairs];
            QaDecode<BITS>::pairs(w[q * (BITS / 4) + k], x);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) r[4 * q + k * kPairs + j] = q_mul2(x[j], fs[k * kPairs + j]);
          }
        }
        tmem_st_32x32b_x16(to + 64 * vb.at + token / 2, r);
      }
    }
    __syncwarp();
    qa_arrive(&sb.empty[st.at], lane);
    tmem_st_wait();
    tc_fence_before_sync();
    __syncwarp();
    qa_arrive(&sb.v_ready[vb.at], lane);
    st.next(C::kTeams);
    vb.next(C::kTeams);
  }
}

// ------------------------------------------------------------------- softmax
// Fragments of 16 lanes x 8 columns: thread i holds row i / 4 in two registers
// and that + 8 in the other two, columns 2 (i % 4) and the next.
__device__ __forceinline__ void qa_load_8(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at));
}
__device__ __forceinline__ void qa_load_16(uint32_t at, uint32_t (&a)[4], uint32_t (&b)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]), "=r"(b[0]), "=r"(b[1]), "=r"(b[2]), "=r"(b[3])
               : "r"(at));
}
// Completes the loads of n fragments; nothing reads the registers before it.
template <int N, int K>
__device__ __forceinline__ void qa_load_wait(uint32_t (&r)[N][K][4]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int k = 0; k < K * N; ++k) {
    uint32_t* x = r[k / K][k % K];
    asm volatile("" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]) : : "memory");
  }
}

// A group of four softmax warps: the only one, or one with 32 of the rows to
// itself.
template <int NMAX>
struct QaGroup {
  static constexpr int kRows = NMAX == 16 ? 16 : 32;
  int lane, w, i;  // of the warp; warp of the group (TMEM lanes 32 w ..), group
  __device__ __forceinline__ QaGroup()
      : lane(threadIdx.x & 31), w((threadIdx.x >> 5) & 3), i(NMAX == 16 ? 0 : threadIdx.x >> 7) {}
  __device__ __forceinline__ int row0() const { return kRows * i; }
  __device__ __forceinline__ int rows(int all) const { return NMAX == 16 ? all : min(max(all - kRows * i, 0), kRows); }
  __device__ __forceinline__ bool vote(bool x) const {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, %2, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"((uint32_t)x), "r"(1 + 2 * i)
        : "memory");
    return any != 0;
  }
  __device__ __forceinline__ void sync() const { named_barrier_sync(2 + 2 * i, 128); }
  __device__ __forceinline__ uint32_t lanes() const { return (uint32_t)(32 * w) << 16; }
};

// Four warps that write O, or a partial result, of each segment that has ended.
template <int D, int BITS, int NMAX>
__device__ void qa_results(const QaParams& p, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  const int lane = threadIdx.x & 31, w = (threadIdx.x >> 5) & 3, d = 32 * w + lane;
#pragma unroll 1
  for (int seg = 0;; ++seg) {
    const int buf = seg & 1;
    if (!qa_wait(&sb.end_ready[buf], (seg >> 1) & 1, wt)) return;
    const int info = sb.last[buf];
    if (info & kQaEnd) return;
    const int4 e0 = sb.segs[seg % kQaSched][0], e1 = sb.segs[seg % kQaSched][1];
    const int rows = qa_rows(info), kind = qa_kind(info);
    const bool direct = e1.z < 0, faulty = info & kQaFaulty;
    const int slot_rows = kind == kQaPrefix ? kQaRows : min(p.rows, kQaRows);
    // A lane has the sums and references of rows `lane` and 32 + lane.
    float inv[(NMAX + 31) / 32];
#pragma unroll
    for (int k = 0; 32 * k < NMAX; ++k) {
      const int n = min(32 * k + lane, NMAX - 1);
      const float(*from)[kQaRows] = sb.sums[buf];
      const float l = from[0][n] + from[1][n] + from[2][n] + from[3][n], top = sb.top[buf][n];
      if (!direct && w == 0 && 32 * k + lane < rows)
        p.work.ml[kind][(size_t)e1.z * slot_rows + n] = faulty ? make_float2(0.0f, NAN) : make_float2(top, l);
      inv[k] = l > 0.0f && !faulty && top > -INFINITY ? 1.0f / l : 0.0f;
    }
    if (!qa_wait(&sb.o_full[buf], (seg >> 1) & 1, wt)) return;
    tc_fence_after_sync();
    if (32 * w < D) {
      float* part = p.work.O[kind] + (size_t)(direct ? 0 : e1.z) * slot_rows * D + d;
      uint16_t* out = reinterpret_cast<uint16_t*>(p.O) +
                      (((size_t)e0.w * p.cache.n_kv_heads + e1.x) * p.rows + e1.y) * D + d;
#pragma unroll 1
      for (int n0 = 0; n0 < rows; n0 += 4, part += 4 * D, out += 4 * D) {
        uint32_t v[4];
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                     : "r"(((uint32_t)(32 * w) << 16) + C::kTmemO + seg % C::kOuts * NMAX + n0));
        asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]) : : "memory");
        const int left = rows - n0;
        if (!direct) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (k < left) part[k * D] = __uint_as_float(v[k]);
        } else {
          const float mine = NMAX == 16 || n0 < 32 ? inv[0] : inv[(NMAX + 31) / 32 - 1];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float f = __shfl_sync(0xffffffffu, mine, (n0 + k) & 31);
            const float x = f == 0.0f ? 0.0f : __uint_as_float(v[k]) * f;
            const uint32_t both = p.fp16 ? qa_pack_half(x, x) : pack_bf16x2(x, x);
            if (k < left) out[k * D] = (uint16_t)both;
          }
        }
      }
    }
    tc_fence_before_sync();
    __syncwarp();
    qa_arrive(&sb.o_free[buf], lane);
  }
}

// S of keys that a row does not see -> -inf.  `key`: of x[0] and x[1]; x[2] and
// x[3] are of the key 8 further.
__device__ __forceinline__ void qa_mask(uint32_t* x, int key, int2 lim) {
  if (key >= lim.x) x[0] = 0xFF800000u;
  if (key >= lim.y) x[1] = 0xFF800000u;
  if (key + 8 >= lim.x) x[2] = 0xFF800000u;
  if (key + 8 >= lim.y) x[3] = 0xFF800000u;
}

// The largest entry of S of each row among this warp's keys, for new references.
template <int NMAX, int H, class Shared>
__device__ __forceinline__ void qa_look(Shared& sb, uint32_t s_at, int pos, int seg, int rows, bool mask) {
  const QaGroup<NMAX> q;
  const int row0 = q.row0(), row_end = row0 + q.rows(rows), lane = q.lane;
#pragma unroll 1
  for (int n0 = row0; n0 < row_end; n0 += 8) {
    uint32_t r[2 * H][1][4];
#pragma unroll
    for (int h = 0; h < 2 * H; ++h)
      qa_load_8(q.lanes() + ((uint32_t)(16 * (h & 1)) << 16) + s_at + (h >> 1) * NMAX + n0, r[h][0]);
    qa_load_wait(r);
    if (mask) {
      const int2 lim = *reinterpret_cast<const int2*>(&sb.lim[seg & 1][n0 + 2 * (lane & 3)]);
#pragma unroll
      for (int h = 0; h < 2 * H; ++h) qa_mask(r[h][0], pos + 32 * q.w + lane / 4 + 128 * (h >> 1) + 16 * (h & 1), lim);
    }
    float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2 * H; ++h) {
      m0 = fmax3(m0, __uint_as_float(r[h][0][0]), __uint_as_float(r[h][0][2]));
      m1 = fmax3(m1, __uint_as_float(r[h][0][1]), __uint_as_float(r[h][0][3]));
    }
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
      m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, x));
      m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, x));
    }
    if (lane < 4) *reinterpret_cast<float2*>(&sb.warp_max[seg & 1][q.w][n0 + 2 * lane]) = make_float2(m0, m1);
  }
}

// The reference of row n, from the largest entries of S that the warps have found.
template <class Shared>
__device__ __forceinline__ float qa_shift(const Shared& sb, int seg, int n) {
  const float(*m)[kQaRows] = sb.warp_max[seg & 1];
  return 7.0f - fmaxf(fmaxf(m[0][n], m[1][n]), fmaxf(m[2][n], m[3][n])) * sb.q_scale[seg & 1][n];
}

// The references at the start of a segment, once the vote has exchanged the
// maxima.  Each warp writes them all, the same, and so needs no barrier.
template <int NMAX, class Shared>
__device__ __forceinline__ bool qa_first(Shared& sb, const QaWait& wt, int seg, int rows, float2* sums) {
  const QaGroup<NMAX> q;
  const int own = q.rows(rows), n = q.row0() + q.lane;
  if (seg >= 2 && !qa_wait(&sb.o_free[seg & 1], ((seg >> 1) - 1) & 1, wt)) return false;
  if (q.lane < q.kRows) {
    float moved = INFINITY;
    // (Rows that see nothing have queries of 0.)
    if (q.lane < own && sb.lim[seg & 1][n] > 0) moved = qa_shift(sb, seg, n);
    sb.top[seg & 1][n] = -moved;
    sb.shift[seg & 1][n] = moved == INFINITY ? 0.0f : moved;
  }
#pragma unroll 1
  for (int n0 = 0; n0 < own; n0 += 8) sums[n0 * 16] = make_float2(0.0f, 0.0f);
  __syncwarp();
  return true;
}

// New references of step t's rows where a numerator passed 2^15.  All four warps
// of a group.  `sums`: this thread's entries of its group's rows, as the step
// before left them.  Returns false when a wait has run out, which the next vote
// will tell.
template <int D, int NMAX, int H, int DEPTH, class Shared>
__device__ __noinline__ bool qa_turn(Shared& sb, const QaWait& wt, uint32_t s_at, uint32_t o_at, int t, int pos,
                                     int seg, int rows, bool mask, float2* sums) {
  const QaGroup<NMAX> q;
  const int row0 = q.row0(), row_end = row0 + q.rows(rows);
  qa_look<NMAX, H>(sb, s_at, pos, seg, rows, mask);
  q.sync();
  const int n = row0 + threadIdx.x % 128;
  if (n < row_end) {
    float moved = INFINITY, f = 1.0f;
    if (sb.lim[seg & 1][n] > 0) {
      const float old = -sb.top[seg & 1][n];
      moved = fminf(old, qa_shift(sb, seg, n));
      if (moved != INFINITY) f = ex2_approx(moved - old);
    }
    sb.top[seg & 1][n] = -moved;
    sb.shift[seg & 1][n] = moved == INFINITY ? 0.0f : moved;
    sb.factor[n] = f;
  }
  q.sync();
#pragma unroll 1
  for (int n0 = row0; n0 < row_end; n0 += 8) {
    float2* l = sums + (n0 - row0) * 16;
    const float2 f = *reinterpret_cast<const float2*>(&sb.factor[n0 + 2 * (q.lane & 3)]);
    *l = make_float2(l->x * f.x, l->y * f.y);
  }
  // O in units of the new references.
  const int u = t - 1;
  if (!qa_wait(&sb.pv_done[u % DEPTH], (u / DEPTH) & 1, wt)) return false;
  if (32 * q.w < D) {
    tc_fence_after_sync();
    const uint32_t at = q.lanes() + o_at;
#pragma unroll 1
    for (int n0 = row0; n0 < row_end; n0 += 4) {
      uint32_t v[4];
      asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                   : "r"(at + n0));
      asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]) : : "memory");
      const float4 f = *reinterpret_cast<const float4*>(&sb.factor[n0]);
      asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at + n0),
                   "r"(__float_as_uint(__uint_as_float(v[0]) * f.x)), "r"(__float_as_uint(__uint_as_float(v[1]) * f.y)),
                   "r"(__float_as_uint(__uint_as_float(v[2]) * f.z)), "r"(__float_as_uint(__uint_as_float(v[3]) * f.w))
                   : "memory");
    }
    tmem_st_wait();
  }
  tc_fence_before_sync();
  return true;
}

// After the last step of a segment: what its results need besides O.  `sums` as
// that step left them.
template <int NMAX, class Shared>
__device__ __forceinline__ void qa_last(Shared& sb, int info, int seg, const float2* sums) {
  const QaGroup<NMAX> q;
  const int buf = seg & 1;
  const int row0 = q.row0(), row_end = row0 + q.rows(qa_rows(info));
#pragma unroll 1
  for (int n0 = row0; n0 < row_end; n0 += 8) {
    float2 l = sums[(n0 - row0) * 16];
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
      l.x += __shfl_xor_sync(0xffffffffu, l.x, x);
      l.y += __shfl_xor_sync(0xffffffffu, l.y, x);
    }
    if (q.lane < 4) *reinterpret_cast<float2*>(&sb.sums[buf][q.w][n0 + 2 * q.lane]) = l;
  }
  if (threadIdx.x == 0) sb.last[buf] = info;
  __syncwarp();
  qa_arrive(&sb.end_ready[buf], q.lane);
}

template <int D, int BITS, int NMAX>
__device__ void qa_softmax(const QaParams& p, uint8_t* p_tiles, float2* all_sums, QA_SHARED& sb, const QaWait& wt) {
  using C = QaCfg<D, BITS, NMAX>;
  const QaGroup<NMAX> q;
  constexpr int H = C::kHalves;
  constexpr int kAt = NMAX == 16 ? 1 : 2;  // groups of 8 rows at a time
  const int lane = q.lane;
  const uint32_t s_at = q.lanes() + C::kTmemS + q.row0();
  // P: row n of 128 bytes in box (key / 64), 16-byte chunk ((key % 64) / 8) ^
  // (n & 7); this lane gives the address of row lane & 7 of matrix lane >> 3.
  const uint32_t p_at = smem_u32(p_tiles) + (q.w >> 1) * C::kBoxBytes + (q.row0() + (lane & 7)) * 128 +
                        ((((q.w & 1) * 4 + (lane >> 3)) ^ (lane & 7)) << 4);
  // Sums: [step & 1][rows / 8][thread]; a step adds to those of the step before.
  float2* const sums = all_sums + q.row0() * 16 + threadIdx.x % 128;
  constexpr int kSumsStep = NMAX / 8 * 128;
  int seg = -1;
  bool ok = true, faulty = false;
  QaRing<C::kDepth> r3;
  // Once a wait of a warp has run out, the next vote ends all; every step has one.
#pragma unroll 1
  for (int t = 0;; ++t, r3.next()) {
    const int b = r3.at, odd = t & 1;
    ok = ok && qa_wait(&sb.s_full[b], r3.phase, wt);
    const int2 e = sb.sched[t % kQaSched];
    const int info = ok ? e.x : kQaEnd, rows = q.rows(qa_rows(info));
    const bool first = info & kQaFirst;  // (not where a wait has run out)
    bool turn = info & (kQaFirst | kQaEnd), turned = false;
    if (first) ++seg;
    tc_fence_after_sync();
    const bool mask = e.y + 128 * H > sb.min_lim[seg & 1];
    if (first)
      qa_look<NMAX, H>(sb, C::kTmemS + b * H * NMAX, e.y, seg, qa_rows(info), mask);
    else if (!ok && lane == 0)
      sb.failed[q.i] = 1;
#pragma unroll 1
    for (;;) {
      if (!turn) {
        // P with the references as they are, and whether a numerator passes 2^15.
        float top = -INFINITY;
#pragma unroll 1
        for (int g2 = 0; 8 * g2 < rows; g2 += kAt) {
          uint32_t r[2 * H][kAt][4];
#pragma unroll
          for (int h = 0; h < 2 * H; ++h) {
            const uint32_t at = s_at + ((uint32_t)(16 * (h & 1)) << 16) + (b * H + (h >> 1)) * NMAX + 8 * g2;
            if constexpr (kAt == 2)
              qa_load_16(at, r[h][0], r[h][1]);
            else
              qa_load_8(at, r[h][0]);
          }
          const int n = q.row0() + 8 * g2 + 2 * (lane & 3);
          const float *shifts = &sb.shift[seg & 1][n], *scales = &sb.q_scale[seg & 1][n];
          float2* const from = sums + (odd ^ 1) * kSumsStep + g2 * 128;
          float2* const to = sums + odd * kSumsStep + g2 * 128;
          float2 scale[kAt], shift[kAt], l[kAt];
#pragma unroll
          for (int k = 0; k < kAt; ++k) {
            scale[k] = *reinterpret_cast<const float2*>(scales + 8 * k);
            shift[k] = *reinterpret_cast<const float2*>(shifts + 8 * k);
            l[k] = from[128 * k];
          }
          qa_load_wait(r);
          if (__builtin_expect(mask, 0)) {
#pragma unroll
            for (int k = 0; k < kAt; ++k) {
              const int2 lim = *reinterpret_cast<const int2*>(&sb.lim[seg & 1][n + 8 * k]);
#pragma unroll
              for (int h = 0; h < 2 * H; ++h)
                qa_mask(r[h][k], e.y + 32 * q.w + lane / 4 + 128 * (h >> 1) + 16 * (h & 1), lim);
            }
          }
#pragma unroll
          for (int k = 0; k < kAt; ++k) {
            float2 part = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int h = 0; h < H; ++h) {
              uint32_t pk[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t* x = r[2 * h + (j >> 1)][k] + 2 * (j & 1);
                const float x0 = fmaf(__uint_as_float(x[0]), scale[k].x, shift[k].x);
                const float x1 = fmaf(__uint_as_float(x[1]), scale[k].y, shift[k].y);
                top = fmax3(top, x0, x1);
                const float a = ex2_approx(x0), c = ex2_approx(x1);
                part.x += a;
                part.y += c;
                pk[j] = qa_pack_half(a, c);
              }
              asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(
                               p_at + b * C::kPBytes + 2 * h * C::kBoxBytes + (g2 + k) * 1024),
                           "r"(pk[0]), "r"(pk[1]), "r"(pk[2]), "r"(pk[3])
                           : "memory");
            }
            to[128 * k] = make_float2(l[k].x + part.x, l[k].y + part.y);
          }
        }
        if (turned) break;
        turn = top > 15.0f;
      }
      if (!q.vote(turn)) break;
      // (A failed warp votes for a turn, and so do all at the start and the end of a segment.)
      if (*reinterpret_cast<volatile int*>(&sb.failed[q.i])) return;
      if (info & kQaEnd) {
        if (seg >= 1 && !qa_wait(&sb.o_free[(seg + 1) & 1], ((seg - 1) >> 1) & 1, wt)) return;
        if (q.w == 0 && q.i == 0 && lane == 0) sb.last[(seg + 1) & 1] = kQaEnd;
        __syncwarp();
        qa_arrive(&sb.end_ready[(seg + 1) & 1], lane);
        return;
      }
      float2* const from = sums + (odd ^ 1) * kSumsStep;
      if (first)
        ok = qa_first<NMAX>(sb, wt, seg, qa_rows(info), from);
      else
        ok = qa_turn<D, NMAX, H, C::kDepth>(sb, wt, C::kTmemS + b * H * NMAX, C::kTmemO + seg % C::kOuts * NMAX, t, e.y,
                                            seg, qa_rows(info), mask, from);
      if (first) faulty = false;
      turn = false;
      turned = true;
    }
    if (info & kQaFaulty) faulty = true;
    tc_fence_before_sync();
    fence_proxy_async_smem();
    __syncwarp();
    qa_arrive(&sb.s_free[b], lane);
    qa_arrive(&sb.p_ready[b], lane);
    if (info & kQaLast) {
      qa_arrive(&sb.q_free[seg & 1], lane);  // the limits have been read
      if (ok) qa_last<NMAX>(sb, faulty ? info | kQaFaulty : info, seg, sums + odd * kSumsStep);
    }
  }
}

// Where the partial results of a unit (request, kv head and row chunk) lie, as
// two int4: {n, n_pre, row of the prefix items, 0}, {first prefix slot, first
// own slot, 0, 0}; n is -1 where O has been written, 0 where nothing is seen.
static __device__ __noinline__ void qa_sources(const QaParams& p, const QaPlan& plan, int unit, int4* out) {
  const int kv = p.cache.n_kv_heads, per = kv * p.chunks;
  const int req = unit / per, rest = unit - req * per, kvh = rest / p.chunks;
  const int g = plan.group[req], tiles = plan.cum[req + 1] - plan.cum[req];
  int n_pre = 0, n_own = 0, row0 = 0, pre_slot = 0, own_slot = 0;
  if (plan.len[req] > 0) {
    if (g >= 0) {
      const int at = req - plan.start[g], tile = at / p.per_tile;
      row0 = (at - tile * p.per_tile) * p.rows;
      const int it = kvh * plan.row_tiles[g] + tile, x = plan.base[g] + it * plan.tiles[g];
      const int k0 = pfx_run_of(plan.t->pre, x);
      n_pre = pfx_run_of(plan.t->pre, x + plan.tiles[g] - 1) - k0 + 1;
      pre_slot = plan.item[g] * kv + it + k0;
    }
    if (tiles > 0) {
      const int x = plan.cum[req] * per + rest * tiles;
      const int k0 = pfx_run_of(plan.t->own, x);
      n_own = pfx_run_of(plan.t->own, x + tiles - 1) - k0 + 1;
      own_slot = unit + k0;
    }
  }
  out[0] = make_int4(g < 0 && n_own == 1 ? -1 : n_pre + n_own, n_pre, row0, 0);
  out[1] = make_int4(pre_slot, own_slot, 0, 0);
}

// -------------------------------------------------------------------- kernel
template <int D, int BITS, int NMAX>
__global__ void __launch_bounds__(QaCfg<D, BITS, NMAX>::kThreads, 1)
    quant_attn_kernel(const __grid_constant__ QaParams p) {
  using C = QaCfg<D, BITS, NMAX>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* q_tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* p_tiles = q_tiles + 2 * C::kQBytes;
  uint8_t* ring = q_tiles + C::kFixed;
  const QaPlan plan = qa_plan(reinterpret_cast<int*>(q_tiles + C::kPlanAt), p.batch, p.n_groups);
  __shared__ QA_SHARED sb;
  static_assert(C::kSmem + sizeof(sb) <= 227 * 1024, "shared memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kOther = C::kThreads / 32 - 4;
  if (threadIdx.x == 0) {
    sb.abort = 0;
    for (int i = 0; i < C::kGroups; ++i) sb.failed[i] = 0;
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(&sb.full[i], 1);
      mbar_init(&sb.empty[i], 8);
    }
    for (int i = 0; i < kQaSched; ++i) {
      mbar_init(&sb.sched_full[i], 1);
      mbar_init(&sb.seg_full[i], 1);
    }
    for (int i = 0; i < C::kKeyBuffers; ++i) {
      mbar_init(&sb.k_ready[i], 4);
      mbar_init(&sb.k_free[i], 1);
    }
    for (int i = 0; i < C::kValueBuffers; ++i) {
      mbar_init(&sb.v_ready[i], 4);
      mbar_init(&sb.v_free[i], 1);
    }
    for (int i = 0; i < C::kDepth; ++i) {
      mbar_init(&sb.p_ready[i], 4 * C::kGroups);
      mbar_init(&sb.s_full[i], 2);
      mbar_init(&sb.s_free[i], 4 * C::kGroups);
      mbar_init(&sb.pv_done[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sb.o_full[i], 1);
      mbar_init(&sb.o_free[i], 4);
      mbar_init(&sb.end_ready[i], 4 * C::kGroups);
      mbar_init(&sb.q_ready[i], 1);
      mbar_init(&sb.q_free[i], 4 * C::kGroups + 1);
      mbar_init(&sb.done[i], 1);
    }
    fence_mbar_init();
  }
  if (warp == kOther + 2) {
    tmem_alloc(&sb.tmem_base, 512);
    tmem_relinquish();
  }
  // Everything above may overlap the previous kernel of the stream.
  griddep_wait();
  tc_fence_before_sync();
  qa_make_plan(p, plan, blockIdx.x == 0);  // ends with a barrier
  tc_fence_after_sync();
  if (threadIdx.x == 0) griddep_launch_dependents();  // the merge waits for this grid's end
  const QaWait wt = {&sb.abort, p.cache.status, p.wait_ns};

  if (warp < 4 * C::kGroups) {
    qa_softmax<D, BITS, NMAX>(p, p_tiles, reinterpret_cast<float2*>(p_tiles + C::kDepth * C::kPBytes), sb, wt);
  } else {
    if (warp < kOther - 4) {
      const int k = warp / 4 - C::kGroups;
      if (k < C::kKeyTeams)
        qa_keys<D, BITS, NMAX>(p, k, ring, sb, wt);
      else
        qa_values<D, BITS, NMAX>(p, k - C::kKeyTeams, ring, sb, wt);
    } else if (warp == kOther) {
      qa_producer<D, BITS, NMAX>(p, ring, sb, wt);
    } else if (warp == kOther + 1) {
      qa_queries<D, BITS, NMAX>(p, plan, q_tiles, sb, wt);
      // Where the merge finds its parts.
      const int units = p.batch * p.cache.n_kv_heads * p.chunks;
      for (int i = blockIdx.x * 32 + lane; i < units; i += gridDim.x * 32)
        qa_sources(p, plan, i, p.work.sources + 2 * (size_t)i);
    } else if (warp == kOther + 2) {
      qa_products_s<D, BITS, NMAX>(p, q_tiles, sb, wt);
    } else if (warp < kOther) {
      qa_results<D, BITS, NMAX>(p, sb, wt);
    } else {
      qa_products_pv<D, BITS, NMAX>(p, p_tiles, sb, wt);
    }
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kOther + 2) {
    tc_fence_after_sync();
    tmem_dealloc(0, 512);
  }
}

// --------------------------------------------------------------------- merge
// Joins the partial results of one unit; blockIdx.y takes a share of its rows.
// A thread owns 4 columns of a row and every parts-th of its parts.
constexpr int kQaMergeThreads = 128;

struct QaMergeShape {
  int rows, parts;  // rows of a block, threads that share an element
};

template <int D>
__global__ void __launch_bounds__(kQaMergeThreads) quant_merge_kernel(const QaParams p, const QaMergeShape sh) {
  extern __shared__ float2 stats[];
  __shared__ float4 sums[kQaMergeThreads];
  __shared__ float part_l[kQaMergeThreads];
  constexpr int kCols = D / 4;
  griddep_launch_dependents();  // what follows waits for this grid's end
  griddep_wait();
  const int unit = blockIdx.x, tid = threadIdx.x;
  const int4 s0 = p.work.sources[2 * (size_t)unit], s1 = p.work.sources[2 * (size_t)unit + 1];
  const int n = s0.x, n_pre = s0.y;
  if (n < 0) return;
  const int chunk = unit % p.chunks, first = blockIdx.y * sh.rows;
  const int left = min(p.rows - chunk * kQaRows, kQaRows) - first;  // rows from this block's first
  const int rows = min(sh.rows, left);
  if (rows <= 0) return;
  const int own_rows = min(p.rows, kQaRows);
  const float2* pre_ml = p.work.ml[kQaPrefix] + (size_t)s1.x * kQaRows + s0.z + first;
  const float2* own_ml = p.work.ml[kQaOwn] + (size_t)s1.y * own_rows + first;
  for (int k = tid; k < n * rows; k += kQaMergeThreads) {
    const int i = k / rows, r = k - i * rows;
    stats[k] = i < n_pre ? pre_ml[(size_t)i * kQaRows + r] : own_ml[(size_t)(i - n_pre) * own_rows + r];
  }
  __syncthreads();
  const int el = kCols * rows;
  const int part = tid / el, e = tid - part * el, row = e / kCols, col = e - row * kCols;
  const bool on = part < sh.parts;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float l = 0.0f;
  if (on) {
    float m = -INFINITY;
    for (int i = 0; i < n; ++i) m = fmaxf(m, stats[i * rows + row].x);
    if (m > -INFINITY) {
      const float4* pre = reinterpret_cast<const float4*>(p.work.O[kQaPrefix]) +
                          ((size_t)s1.x * kQaRows + s0.z + first + row) * kCols + col;
      const float4* own = reinterpret_cast<const float4*>(p.work.O[kQaOwn]) +
                          ((size_t)s1.y * own_rows + first + row) * kCols + col;
#pragma unroll 4
      for (int i = part; i < n; i += sh.parts) {
        const float4 v = i < n_pre ? pre[(size_t)i * kQaRows * kCols] : own[(size_t)(i - n_pre) * own_rows * kCols];
        const float2 st = stats[i * rows + row];
        if (st.x == -INFINITY) continue;  // the row saw nothing there
        const float u = ex2_approx(st.x - m);
        l += st.y * u;
        acc.x += u * v.x;
        acc.y += u * v.y;
        acc.z += u * v.z;
        acc.w += u * v.w;
      }
    }
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
  if (part > 0) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;  // 0 as well where a faulty page made l NaN
  if (inv == 0.0f) acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const size_t out_row = (size_t)(unit / p.chunks) * p.rows + chunk * kQaRows + first + row;
  uint2 out;
  if (p.fp16)
    out = make_uint2(qa_pack_half(acc.x * inv, acc.y * inv), qa_pack_half(acc.z * inv, acc.w * inv));
  else
    out = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  reinterpret_cast<uint2*>(p.O)[out_row * kCols + col] = out;
}

template <int D, int BITS, int NMAX>
cudaError_t launch_quant_attn_instance(QaLaunch L) {
  using C = QaCfg<D, BITS, NMAX>;
  auto kern = quant_attn_kernel<D, BITS, NMAX>;
  L.p.keys = 128 * C::kHalves;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(L.grid);
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = L.stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if ((e = cudaLaunchKernelEx(&cfg, kern, L.p)) != cudaSuccess) return e;
  // Rows of a block: as many as it has threads for, fewer (the threads then
  // share elements) while the blocks are few.
  const int rows = L.p.rows < kQaRows ? L.p.rows : kQaRows;
  const long long units = (long long)L.p.batch * L.p.cache.n_kv_heads * L.p.chunks;
  QaMergeShape sh;
  sh.rows = kQaMergeThreads / (D / 4);
  if (sh.rows > rows) sh.rows = rows;
  while (sh.rows > 1 && units * ((rows + sh.rows - 1) / sh.rows) < 8 * L.grid) sh.rows = (sh.rows + 1) / 2;
  sh.parts = kQaMergeThreads / (D / 4 * sh.rows);
  cfg.gridDim = dim3((unsigned)units, (rows + sh.rows - 1) / sh.rows);
  cfg.blockDim = dim3(kQaMergeThreads);
  cfg.dynamicSmemBytes = (size_t)(2 * L.grid + 2) * sh.rows * sizeof(float2);
  return cudaLaunchKernelEx(&cfg, quant_merge_kernel<D>, L.p, sh);
}

template <int D>
cudaError_t launch_quant_attn_for_dim(const QaLaunch& L) {
  if (L.p.cache.bits == 4)
    return L.wide ? launch_quant_attn_instance<D, 4, 64>(L) : launch_quant_attn_instance<D, 4, 16>(L);
  return L.wide ? launch_quant_attn_instance<D, 8, 64>(L) : launch_quant_attn_instance<D, 8, 16>(L);
}

}  // namespace wise
