// The paged cache's own operations: forking sequences, growing them (page
// allocation and copy-on-write), storing new keys and values, dropping tokens
// and closing up the pages in use.  All state is integers in device memory;
// every result is a function of the inputs alone, whatever order the threads
// run in: pages are taken and moved by rank (prefix sums over refs), and the
// atomics below are integer additions and ORs whose order does not show.
#include <cooperative_groups.h>

#include <algorithm>

#include "cache_common.cuh"
#include "ptx.cuh"

namespace wise {
namespace {

namespace cg = cooperative_groups;

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;

// ---------------------------------------------------------------------- fork
// One block per entry.  An entry whose dst occurs again in a used entry is
// left out, so no two blocks touch the same row.  Both rows are looked through
// before anything changes.  Bound by its chain of dependent accesses (list,
// length, table, count) and the launch.
__global__ void __launch_bounds__(256) fork_kernel(const CacheView c, const int32_t* src, const int32_t* dst, int n) {
  const int i = blockIdx.x;
  const int s = src[i], d = dst[i];
  if (s < 0 || d < 0) return;
  int bad = s >= c.n_slots || d >= c.n_slots;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const int sj = src[j], dj = dst[j];
    if (sj >= 0 && dj >= 0 && ((j != i && dj == d) || sj == d)) bad = 1;
  }
  int len = 0, old = 0;
  if (s < c.n_slots && d < c.n_slots) {
    len = c.lens[s];
    old = c.lens[d];
    if (len < 0 || len > c.max_len || old < 0 || old > c.max_len) bad = 1;
  }
  const int32_t* from = c.table + (size_t)s * c.max_pages;
  int32_t* to = c.table + (size_t)d * c.max_pages;
  if (!bad) {
    for (int k = threadIdx.x; k < pages_of(c, old); k += blockDim.x) bad |= !valid_page(c, to[k]);
    for (int k = threadIdx.x; k < pages_of(c, len); k += blockDim.x) bad |= !valid_page(c, from[k]);
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) fault(c, kStatusBadCache);
    return;
  }
  for (int k = threadIdx.x; k < pages_of(c, old); k += blockDim.x) atomicAdd(c.refs + to[k], -1);
  for (int k = threadIdx.x; k < pages_of(c, len); k += blockDim.x) {
    const int page = from[k];
    atomicAdd(c.refs + page, 1);
    to[k] = page;
  }
  if (threadIdx.x == 0) c.lens[d] = len;  // every thread read it before the barrier
}

// ---------------------------------------------------------------------- drop
// One block per entry, and bound like a fork; the pages are looked through before
// anything changes.
__global__ void __launch_bounds__(256) drop_kernel(const CacheView c, const int32_t* slots, const int32_t* n_drop,
                                                   int n) {
  const int i = blockIdx.x;
  const int s = slots[i];
  if (s < 0) return;
  const int drop = n_drop[i];
  int bad = s >= c.n_slots || drop < 0;
  for (int j = threadIdx.x; j < n; j += blockDim.x)
    if (j != i && slots[j] == s) bad = 1;
  int len = 0;
  if (s < c.n_slots) {
    len = c.lens[s];
    if (len < 0 || len > c.max_len) bad = 1;
  }
  const int left = max(len - max(drop, 0), 0);
  const int32_t* row = c.table + (size_t)s * c.max_pages;
  if (!bad)
    for (int k = pages_of(c, left) + threadIdx.x; k < pages_of(c, len); k += blockDim.x)
      bad |= !valid_page(c, row[k]);
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) fault(c, kStatusBadCache);
    return;
  }
  for (int k = pages_of(c, left) + threadIdx.x; k < pages_of(c, len); k += blockDim.x)
    atomicAdd(c.refs + row[k], -1);
  if (threadIdx.x == 0) c.lens[s] = left;
}

// -------------------------------------------------------------------- extend
// Sums of page counts stop at kSumCap, above every n_pages, so that absurd
// lists cannot wrap them around (the capped sum is still associative).
constexpr int kSumCap = (1 << 30) - 1;
__device__ __forceinline__ int capped_sum(int a, int b) { return min(a + b, kSumCap); }

// Inclusive prefix sum over the block; `total` receives the block's sum.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v = capped_sum(v, t);
  }
  if (lane == 31) warp_sums[w] = v;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int k = 0; k < kPlanThreads / 32; ++k) {
    const int t = warp_sums[k];
    if (k < w) before = capped_sum(before, t);
    total = capped_sum(total, t);
  }
  __syncthreads();
  return capped_sum(v, before);
}

// Ranks of the pages in use, over one cluster of 1 or 8 blocks.  A warp owns a
// contiguous part of refs and passes over it twice, coalesced: once to count,
// once (after the sums have been exchanged through distributed shared memory)
// to hand each page its rank.
struct PageScan {
  int v0, v1;   // this warp's pages
  int before;   // pages in use below v0
  int total;    // pages in use
};
constexpr int kScanUnroll = 8;

__device__ __forceinline__ int count_used(const CacheView& c, int v0, int v1, int lane) {
  int n = 0;
  for (int base = v0 + lane; base < v1; base += 32 * kScanUnroll) {
    int r[kScanUnroll];
#pragma unroll
    for (int k = 0; k < kScanUnroll; ++k) r[k] = base + 32 * k < v1 ? c.refs[base + 32 * k] : 0;
#pragma unroll
    for (int k = 0; k < kScanUnroll; ++k) n += r[k] != 0;
  }
  return __reduce_add_sync(0xffffffffu, n);
}

// All threads of the cluster; `sums` (kPlanWarps ints) and `block_sum` are
// shared memory.  The first pass; ends with a cluster barrier.
__device__ __forceinline__ PageScan scan_pages(const CacheView& c, const cg::cluster_group& cluster, int* sums,
                                               int* block_sum) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int n_warps = cluster.num_blocks() * kPlanWarps;
  const int part = (c.n_pages + n_warps - 1) / n_warps;
  PageScan s;
  s.v0 = (int)min((long long)(cluster.block_rank() * kPlanWarps + w) * part, (long long)c.n_pages);
  s.v1 = min(s.v0 + part, c.n_pages);
  const int n = count_used(c, s.v0, s.v1, lane);
  if (lane == 0) sums[w] = n;
  __syncthreads();
  if (w == 0) {
    const int all = __reduce_add_sync(0xffffffffu, sums[lane]);
    if (lane == 0) *block_sum = all;
  }
  cluster.sync();
  s.before = 0;
  s.total = 0;
  for (int k = 0; k < (int)cluster.num_blocks(); ++k) {
    const int t = *cluster.map_shared_rank(block_sum, k);
    if (k < (int)cluster.block_rank()) s.before += t;
    s.total += t;
  }
  const int mine = lane < w ? sums[lane] : 0;
  s.before += __reduce_add_sync(0xffffffffu, mine);
  return s;
}

// The second pass: visit(page, in use, pages in use below it) for the warp's pages.
template <class Visit>
__device__ __forceinline__ void visit_pages(const CacheView& c, const PageScan& s, Visit visit) {
  const int lane = threadIdx.x & 31;
  int before = s.before;
  for (int base = s.v0; base < s.v1; base += 32 * kScanUnroll) {
    int r[kScanUnroll];
#pragma unroll
    for (int k = 0; k < kScanUnroll; ++k) {
      const int page = base + 32 * k + lane;
      r[k] = page < s.v1 ? c.refs[page] : 0;
    }
#pragma unroll
    for (int k = 0; k < kScanUnroll; ++k) {
      const int page = base + 32 * k + lane;
      const uint32_t used = __ballot_sync(0xffffffffu, r[k] != 0);
      if (page < s.v1) visit(page, r[k] != 0, before + __popc(used & ((1u << lane) - 1u)));
      before += __popc(used);
    }
  }
}

// Blocks of a plan: one up to 4096 pages, where a block's two passes take no
// longer than the cluster's barriers.  (64 sequences grown by a page and cut
// again, and an empty compaction, with one block and with eight: 1000 pages 11.4
// and 6.2 us, 11.7 and 6.4; 4000 pages 11.9 and 6.7, 11.9 and 6.6; 8000 pages
// 12.4 and 7.3, 12.3 and 6.7; 64000 pages 20.3 and 18.0, 12.7 and 7.4.)
inline int plan_blocks(const CacheView& c) { return c.n_pages <= 4096 ? 1 : 8; }

// Workspace words: [0] number of copies; then the free list, the entries'
// needs, and the copies as (from, to, rows).
struct ExtendWork {
  int32_t* count;
  int32_t* free_ids;
  int32_t* need;
  int32_t* copies;
};
__host__ __device__ inline ExtendWork extend_work(int32_t* w, int n_pages, int n) {
  ExtendWork e;
  e.count = w;
  e.free_ids = w + 4;
  e.need = e.free_ids + n_pages;
  e.copies = e.need + n;
  return e;
}
constexpr int kNeedCopy = 1 << 30;  // flag beside an entry's number of pages
constexpr int kNeedNone = -1;       // unused or faulty entry

// One cluster.  Block 0 finds the need of every entry from the state before
// the call while all of them count the pages in use; then the lowest free
// pages are listed, as many as are needed, and block 0 assigns them.
__global__ void __launch_bounds__(kPlanThreads) extend_plan_kernel(const CacheView c, const int32_t* slots,
                                                                   const int32_t* n_new, int n, int32_t* granted,
                                                                   int32_t* work) {
  extern __shared__ uint32_t seen[];  // two bitmaps over the slots: listed, listed twice
  __shared__ int warp_sums[kPlanWarps], scan_sums[kPlanWarps];
  __shared__ int block_used, total_want, n_copies;
  const cg::cluster_group cluster = cg::this_cluster();
  const bool lead = cluster.block_rank() == 0;
  const ExtendWork w = extend_work(work, c.n_pages, n);
  griddep_launch_dependents();  // the copies wait for this grid's end
  if (lead) {
    if (threadIdx.x == 0) n_copies = 0;
    const uint32_t* twice = mark_twice(c, slots, n, seen);
    int want = 0;
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
      const int s = slots[i], add = n_new[i];
      int need = kNeedNone;
      if (s >= 0) {
        const bool in = s < c.n_slots;
        const int len = in ? c.lens[s] : -1;
        if (!in || add < 0 || ((twice[s >> 5] >> (s & 31)) & 1u) || len < 0 || len > c.max_len) {
          fault(c, kStatusBadCache);
        } else if (add > c.max_len - len) {
          fault(c, kStatusNoPages);
        } else {
          need = pages_of(c, len + add) - pages_of(c, len);
          if (add > 0 && len % c.page != 0) {
            const int tail = c.table[(size_t)s * c.max_pages + len / c.page];
            if (!valid_page(c, tail)) {
              fault(c, kStatusBadCache);
              need = kNeedNone;
            } else if (c.refs[tail] > 1) {
              need = (need + 1) | kNeedCopy;
            }
          }
        }
      }
      w.need[i] = need;
      if (need != kNeedNone) want = capped_sum(want, need & ~kNeedCopy);
    }
    int t;
    block_scan(want, warp_sums, t);
    if (threadIdx.x == 0) total_want = t;
  }
  const PageScan scan = scan_pages(c, cluster, scan_sums, &block_used);
  const int wanted = *cluster.map_shared_rank(&total_want, 0);
  const int found = min(wanted, c.n_pages - scan.total);
  if (scan.v0 - scan.before < found)  // a free page of this warp's is among the first
    visit_pages(c, scan, [&](int page, bool used, int below) {
      if (!used && page - below < found) w.free_ids[page - below] = page;
    });
  cluster.sync();  // the list is complete, and the blocks' sums have been read
  if (!lead) return;
  // Assignment, in list order.
  int carry = 0;
  for (int base = 0; base < n; base += kPlanThreads) {
    const int i = base + threadIdx.x;
    const int info = i < n ? w.need[i] : kNeedNone;
    const int need = info == kNeedNone ? 0 : info & ~kNeedCopy;
    int t;
    const int upto = block_scan(need, warp_sums, t);
    if (i < n) {
      const int s = slots[i], add = n_new[i];
      const int end = capped_sum(carry, upto), first = end - need;
      int give = 0;
      if (info != kNeedNone) {
        if (need == 0 || end <= found) {
          give = add;
          const int len = c.lens[s];
          int32_t* row = c.table + (size_t)s * c.max_pages;
          int k = pages_of(c, len);
          if (info & kNeedCopy) {
            --k;
            const int tail = row[k];
            atomicAdd(c.refs + tail, -1);
            const int at = atomicAdd(&n_copies, 1);
            w.copies[3 * at] = tail;
            w.copies[3 * at + 1] = w.free_ids[first];
            w.copies[3 * at + 2] = len % c.page;
          }
          for (int j = 0; j < need; ++j) {
            const int page = w.free_ids[first + j];
            row[k + j] = page;
            c.refs[page] = 1;
          }
          c.lens[s] = len + add;
        } else {
          fault(c, kStatusNoPages);
        }
      }
      granted[i] = give;
    }
    carry = capped_sum(carry, t);
  }
  __syncthreads();
  if (threadIdx.x == 0) *w.count = n_copies;
}

// Copies the first `rows` rows of every head of a page, in every plane; one
// block per (copy, plane, head) in turn, whose rows are contiguous (in 8 and 4
// bits the tokens of a page lie beside one another: all of them).  What
// bounds it: memory for many copies (124 part-filled pages of 8 layers, 146 MB
// written and as much read, most of it from L2, in 21 us).
__global__ void __launch_bounds__(256) copy_tails_kernel(const CacheView c, int32_t* work, int n) {
  griddep_wait();
  const ExtendWork w = extend_work(work, c.n_pages, n);
  const long long jobs = (long long)*w.count * c.n_planes * c.n_kv_heads;
  for (long long job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int head = (int)(job % c.n_kv_heads);
    const long long r = job / c.n_kv_heads;
    const int plane = (int)(r % c.n_planes), at = (int)(r / c.n_planes);
    uint8_t* base = c.pool + plane * c.plane_bytes + (size_t)head * c.head_bytes;
    const uint4* from = reinterpret_cast<const uint4*>(base + (size_t)w.copies[3 * at] * c.page_bytes);
    uint4* to = reinterpret_cast<uint4*>(base + (size_t)w.copies[3 * at + 1] * c.page_bytes);
    const int units = c.bits == 16 ? w.copies[3 * at + 2] * (c.row_bytes / 16) : c.head_bytes / 16;
    for (int k = threadIdx.x; k < units; k += blockDim.x) to[k] = from[k];
  }
}

// --------------------------------------------------------------------- write
// One thread per 16 bytes of K or of V (blockIdx.y = 0, 1); a block takes pieces
// of kRows rows in turn.  Two entries of one slot would store to the same places
// in any order, so each block first marks the slots that the list has twice;
// there are no more blocks than stay resident, so that this work grows with the
// list only.  What bounds it: for a few tokens the chain slot, length, page, count
// before the store (640 tokens of 8 heads of 128, 5 MB: about 4 us), so the value
// is loaded beside it; for prompts memory (64 x 4096 tokens of 8 heads of 128:
// 341 us, 6.3 TB/s; with a block for every piece, which cannot afford the marks,
// 430).  For 1024 sequences grown by a token a write takes 8.0 us, 7.7 without
// the marks; for 16384, 22 and 7.7.
template <int PER_ROW>
__global__ void __launch_bounds__(256, 8) write_kernel(const CacheView c, int layer, const int32_t* slots,
                                                       const int32_t* n_new, int batch, int q_len, int rows,
                                                       const uint4* K, const uint4* V) {
  extern __shared__ uint32_t seen[];
  constexpr int kRows = 256 / PER_ROW;
  const int in_piece = threadIdx.x / PER_ROW, unit = threadIdx.x % PER_ROW;
  const uint4* from = blockIdx.y ? V : K;
  uint8_t* plane = c.pool + (2 * layer + blockIdx.y) * c.plane_bytes;
  const uint32_t* twice = batch > 1 ? mark_twice(c, slots, batch, seen) : nullptr;
  if (in_piece >= kRows) return;
  for (int r = blockIdx.x * kRows + in_piece; r < rows; r += gridDim.x * kRows) {
    // On its way while the page is looked up.
    const uint4 value = from[(size_t)r * PER_ROW + unit];
    const int bh = r / q_len, i = r - bh * q_len;
    const int b = bh / c.n_kv_heads, head = bh - b * c.n_kv_heads;
    const int s = slots[b], add = n_new ? n_new[b] : q_len;
    if (s < 0) continue;
    const bool in = s < c.n_slots && !(twice && ((twice[s >> 5] >> (s & 31)) & 1u));
    const int len = in ? c.lens[s] : -1;
    if (len < 0 || len > c.max_len || add < 0 || add > q_len || add > len) {
      fault(c, kStatusBadCache);
      continue;
    }
    if (i >= add) continue;
    const int pos = len - add + i;
    const int page = c.table[(size_t)s * c.max_pages + (pos >> c.page_shift)];
    if (!valid_page(c, page) || c.refs[page] > 1) {
      fault(c, kStatusBadCache);
      continue;
    }
    uint8_t* to = plane + (size_t)page * c.page_bytes + (size_t)head * c.head_bytes +
                  (size_t)(pos & (c.page - 1)) * c.row_bytes;
    reinterpret_cast<uint4*>(to)[unit] = value;
  }
}

// ------------------------------------------------------------------- compact
// Workspace words: [0] number of moves; then the holes below n_live ascending,
// and the pages that move into them descending.
//
// With u(g) = the pages in use below page g: a hole g has rank g - u(g) among
// the free pages, hence among the holes; a page in use g >= n_live comes
// n_live - 1 - u(g) places before the last one; and the number of moves is
// n_live - u(n_live).
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(const CacheView c, int32_t* remap,
                                                                    int32_t* n_live_out, int32_t* work) {
  __shared__ int scan_sums[kPlanWarps];
  __shared__ int block_used;
  const cg::cluster_group cluster = cg::this_cluster();
  griddep_launch_dependents();  // the moves wait for this grid's end
  int32_t* holes = work + 4;
  int32_t* movers = holes + c.n_pages;
  const PageScan scan = scan_pages(c, cluster, scan_sums, &block_used);
  const int n_live = scan.total;
  visit_pages(c, scan, [&](int page, bool used, int below) {
    if (page < n_live) {
      remap[page] = used ? page : -1;
      if (!used) holes[page - below] = page;
    } else if (used) {
      movers[n_live - 1 - below] = page;
    } else {
      remap[page] = -1;
    }
    if (page == n_live) work[0] = n_live - below;
  });
  if (cluster.block_rank() == 0 && threadIdx.x == 0) {
    *n_live_out = n_live;
    if (n_live == c.n_pages) work[0] = 0;  // no page lies past them
  }
  cluster.sync();
  const int n_moves = *reinterpret_cast<volatile int32_t*>(work);
  for (int k = cluster.block_rank() * kPlanThreads + threadIdx.x; k < n_moves; k += cluster.num_blocks() * kPlanThreads) {
    const int from = movers[n_moves - 1 - k], to = holes[k];
    remap[from] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
}

// Moves pages (sources lie at or past n_live, destinations below it, so the
// copies are independent) and renames the tables' entries.  A job is 16 KB of a
// page in one plane, so that a few large pages still fill the GPU.  What bounds
// it: memory (0.68 GB read and as much written in 219 us, 6.2 TB/s).
__global__ void __launch_bounds__(256) compact_move_kernel(const CacheView c, const int32_t* remap,
                                                           const int32_t* work) {
  griddep_wait();
  const int32_t* holes = work + 4;
  const int32_t* movers = holes + c.n_pages;
  const int n_moves = work[0];
  constexpr int kPiece = 16384;  // bytes of a page one block copies at a time
  const int pieces = (c.page_bytes + kPiece - 1) / kPiece;
  const long long jobs = (long long)n_moves * c.n_planes * pieces;
  for (long long job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int piece = (int)(job % pieces);
    const long long r = job / pieces;
    const int plane = (int)(r % c.n_planes), at = (int)(r / c.n_planes);
    uint8_t* base = c.pool + plane * c.plane_bytes + (size_t)piece * kPiece;
    const uint4* from = reinterpret_cast<const uint4*>(base + (size_t)movers[n_moves - 1 - at] * c.page_bytes);
    uint4* to = reinterpret_cast<uint4*>(base + (size_t)holes[at] * c.page_bytes);
    const int units = min(kPiece, c.page_bytes - piece * kPiece) / 16;
    for (int k = threadIdx.x; k < units; k += blockDim.x) to[k] = from[k];
  }
  for (int s = blockIdx.x; s < c.n_slots; s += gridDim.x) {
    const int len = c.lens[s];
    if (len < 0 || len > c.max_len) {
      if (threadIdx.x == 0) fault(c, kStatusBadCache);
      continue;
    }
    int32_t* row = c.table + (size_t)s * c.max_pages;
    for (int k = threadIdx.x; k < pages_of(c, len); k += blockDim.x) {
      const int page = row[k];
      if (!valid_page(c, page)) {
        fault(c, kStatusBadCache);
        continue;
      }
      const int to = remap[page];
      if (to < 0)
        fault(c, kStatusBadCache);  // a sequence holds a page that refs calls free
      else if (to != page)
        row[k] = to;
    }
  }
}

}  // namespace

cudaError_t launch_kv_fork(const CacheView& c, const int32_t* src, const int32_t* dst, int n, cudaStream_t stream) {
  fork_kernel<<<n, 256, 0, stream>>>(c, src, dst, n);
  return cudaGetLastError();
}

cudaError_t launch_kv_drop(const CacheView& c, const int32_t* slots, const int32_t* n_drop, int n,
                           cudaStream_t stream) {
  drop_kernel<<<n, 256, 0, stream>>>(c, slots, n_drop, n);
  return cudaGetLastError();
}

// A kernel that waits for the previous one itself (griddep_wait).
template <class... Args>
static cudaError_t launch_dependent(void (*kernel)(Args...), int grid, int threads, cudaStream_t stream, Args... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <class... Args>
static cudaError_t launch_plan(void (*kernel)(Args...), int blocks, int smem, cudaStream_t stream, Args... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

cudaError_t launch_kv_extend(const CacheView& c, const int32_t* slots, const int32_t* n_new, int n, int32_t* granted,
                             int32_t* work, int sm_count, cudaStream_t stream) {
  const int smem = 2 * ((c.n_slots + 31) / 32) * 4;
  cudaError_t e = cudaSuccess;
  // The limit is the kernel's, not the launch's: always the largest one, so that
  // calls of other threads cannot lower it before this launch.
  if (smem > 40 * 1024)
    e = cudaFuncSetAttribute(extend_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlots / 32 * 2 * 4);
  if (e == cudaSuccess)
    e = launch_plan(extend_plan_kernel, plan_blocks(c), smem, stream, c, slots, n_new, n, granted, work);
  if (e != cudaSuccess) return e;
  return launch_dependent(copy_tails_kernel, sm_count * 8, 256, stream, c, work, n);
}

template <int PER_ROW>
static cudaError_t launch_write(const CacheView& c, int layer, const int32_t* slots, const int32_t* n_new, int batch,
                                int q_len, const void* K, const void* V, int sm_count, cudaStream_t stream) {
  const int rows = batch * c.n_kv_heads * q_len, piece = 256 / PER_ROW;
  const int smem = batch > 1 ? 2 * ((c.n_slots + 31) / 32) * 4 : 0;
  if (smem > 40 * 1024) {
    cudaError_t e = cudaFuncSetAttribute(write_kernel<PER_ROW>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         kMaxSlots / 32 * 2 * 4);
    if (e != cudaSuccess) return e;
  }
  const int blocks = std::min((rows - 1) / piece + 1, 4 * sm_count);  // of K, and as many of V: 8 an SM
  write_kernel<PER_ROW><<<dim3(blocks, 2), 256, smem, stream>>>(c, layer, slots, n_new, batch, q_len, rows,
                                                               reinterpret_cast<const uint4*>(K),
                                                               reinterpret_cast<const uint4*>(V));
  return cudaGetLastError();
}

cudaError_t launch_kv_write(const CacheView& c, int layer, const int32_t* slots, const int32_t* n_new, int batch,
                            int q_len, const void* K, const void* V, int sm_count, cudaStream_t stream) {
  switch (c.row_bytes / 16) {
    case 8: return launch_write<8>(c, layer, slots, n_new, batch, q_len, K, V, sm_count, stream);
    case 12: return launch_write<12>(c, layer, slots, n_new, batch, q_len, K, V, sm_count, stream);
    default: return launch_write<16>(c, layer, slots, n_new, batch, q_len, K, V, sm_count, stream);
  }
}

cudaError_t launch_kv_compact(const CacheView& c, int32_t* remap, int32_t* n_live, int32_t* work, int sm_count,
                              cudaStream_t stream) {
  cudaError_t e = launch_plan(compact_plan_kernel, plan_blocks(c), 0, stream, c, remap, n_live, work);
  if (e != cudaSuccess) return e;
  return launch_dependent(compact_move_kernel, sm_count * 8, 256, stream, c, (const int32_t*)remap,
                          (const int32_t*)work);
}

}  // namespace wise
