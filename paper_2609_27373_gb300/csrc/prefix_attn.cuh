// Attention of new tokens over the paged cache (wise_prefix_attn): types shared
// by the kernel instances, the merge of their partial results and the launch.
//
// Mathematics.  A query row's softmax over its keys is computed part by part:
// a part (a run of key tiles) gives m = the largest logit in base-2 units, l =
// the sum of 2^(s - m) and O = the sum of 2^(s - m) v, all fp32, and parts
// join as  O = sum_k 2^(m_k - M) O_k / sum_k 2^(m_k - M) l_k,  M = max m_k.
//
// Work.  With R = q_len * n_heads / n_kv_heads query rows a request and kv
// head, the tensor cores take tiles of 128 rows x 128 keys.  Three kinds of
// items exist, each for one kv head:
//   pair    the shared prefix of a group against two tiles of floor(128 / R)
//           requests each: every key tile that is loaded serves both;
//   single  the same against the odd tile that is left (or the only one);
//   own     one request's keys past the shared prefix, R rows of the tile.
// A CTA holds two streams, each a softmax warpgroup with its own S, P and O in
// tensor memory and its own MMA-issuing thread.  A pair item occupies both on
// the same key tiles; single and own items occupy one each.  The key tiles of
// all pair items form one line that is cut into equal runs, one a CTA, and
// those of all other items another, cut into equal runs, one a stream.  So
// every CTA gets the same number of tiles whatever the lengths are, long
// sequences are split over many CTAs, and the cuts depend on nothing but the
// lengths and the number of SMs (results repeat bit for bit).  A (run, item)
// overlap is a segment; its partial result goes to the workspace slot
// item + run, which is unique because both only grow along the line.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "internal.cuh"

namespace wise {

constexpr int kPfxMaxBatch = 1024;
constexpr int kPfxMaxGroups = 256;
constexpr int kPfxRows = 128;  // query rows of a tile
constexpr int kPfxKeys = 128;  // keys of a tile

enum PfxKind : int { kPfxOwn = 0, kPfxSingle = 1, kPfxPair = 2 };

// A line of tiles cut into runs of q or q + 1 tiles, the longer ones (`longer`
// of them) first: where run k starts, and the run that holds tile x.
struct PfxCuts {
  int runs, q, longer;
};
__host__ __device__ inline PfxCuts pfx_cuts(int tiles, int max_runs) {
  PfxCuts c;
  c.runs = tiles < max_runs ? tiles : max_runs;
  c.q = c.runs > 0 ? tiles / c.runs : 0;
  c.longer = tiles - c.q * c.runs;
  return c;
}
__host__ __device__ inline int pfx_cut(const PfxCuts& c, int k) { return k * c.q + (k < c.longer ? k : c.longer); }
__host__ __device__ inline int pfx_run_of(const PfxCuts& c, int x) {
  const int y = x - c.longer * (c.q + 1);
  return y < 0 ? x / (c.q + 1) : c.longer + y / c.q;
}

// The plan of a launch, which every CTA derives in shared memory.  Lists are
// ints.
struct PfxTotals {
  PfxCuts pair;      // the line of pair items
  PfxCuts line;      // the other line: single items first, then own items
  int single_tiles;  // tiles of the single items
  int pad;
};

struct PfxPlan {
  PfxTotals* t;
  // Per request.
  int* slot;   // of the cache
  int* len;    // positions of its sequence, 0 for an unused or faulty request
  int* lo;     // positions read through its group
  int* add;    // new tokens
  int* group;  // index, -1 outside every group with a shared prefix
  int* cum;    // [batch + 1] own tiles (of one kv head) before it
  // Per group.
  int* start;        // [n_groups + 1]
  int* lead;         // first active member
  int* tiles;        // key tiles of the shared prefix, 0 if nothing is shared
  int* pairs;        // pairs of row tiles
  // One after the other, [n_groups + 1] each: sums over the groups before.
  int* pair_base;    // pair tiles
  int* pair_item;    // pair items of one kv head
  int* single_base;  // single tiles
  int* single_item;  // single items of one kv head
};

__host__ __device__ inline int pfx_plan_ints(int batch, int n_groups) {
  return 8 + 6 * batch + 1 + 8 * n_groups + 5;
}

__host__ __device__ inline PfxPlan pfx_plan(int* base, int batch, int n_groups) {
  PfxPlan p;
  p.t = reinterpret_cast<PfxTotals*>(base);
  p.slot = base + 8;
  p.len = p.slot + batch;
  p.lo = p.len + batch;
  p.add = p.lo + batch;
  p.group = p.add + batch;
  p.cum = p.group + batch;
  p.start = p.cum + batch + 1;
  p.lead = p.start + n_groups + 1;
  p.tiles = p.lead + n_groups;
  p.pairs = p.tiles + n_groups;
  p.pair_base = p.pairs + n_groups;
  p.pair_item = p.pair_base + n_groups + 1;
  p.single_base = p.pair_item + n_groups + 1;
  p.single_item = p.single_base + n_groups + 1;
  return p;
}

// Workspace: where the merge finds its parts (two int4 per request and kv
// head), then for each kind its segments' (m, l) pairs and their O, transposed
// as [segment][head_dim / 4][rows][4] so that neighbouring threads (rows) store
// neighbouring 16 bytes.  A pair segment is two slots.
struct PfxWork {
  int4* sources;
  float2* ml[3];
  float4* O[3];
  int rows[3];  // rows of a slot
  size_t bytes;
};

inline PfxWork pfx_work(void* base, int batch, int n_groups, int n_kv_heads, int rows, int head_dim, int sm_count) {
  PfxWork w;
  const int per_tile = kPfxRows / rows;  // requests of a tile
  // A group of m requests has floor(ceil(m / per_tile) / 2) <= m / per_tile
  // pairs, so all groups together at most batch / per_tile.
  const long long slots[3] = {
      (long long)batch * n_kv_heads + 2 * sm_count,
      n_groups ? (long long)n_groups * n_kv_heads + 2 * sm_count : 0,
      n_groups ? 2 * ((long long)(batch / per_tile) * n_kv_heads + sm_count) : 0,
  };
  w.rows[kPfxOwn] = rows;
  w.rows[kPfxSingle] = w.rows[kPfxPair] = kPfxRows;
  uint8_t* at = reinterpret_cast<uint8_t*>(base);
  size_t off = 0;
  auto take = [&](size_t n) {
    uint8_t* p = at + off;
    off += (n + 255) / 256 * 256;
    return p;
  };
  w.sources = reinterpret_cast<int4*>(take((size_t)batch * n_kv_heads * 2 * sizeof(int4)));
  for (int k = 0; k < 3; ++k) w.ml[k] = reinterpret_cast<float2*>(take(slots[k] * w.rows[k] * sizeof(float2)));
  for (int k = 0; k < 3; ++k) w.O[k] = reinterpret_cast<float4*>(take(slots[k] * w.rows[k] * head_dim * 4));
  w.bytes = off;
  return w;
}

struct PfxParams {
  CacheView cache;
  int batch, q_len, n_heads, group, n_groups, rows, per_tile;
  float scale_log2;
  const int32_t* slots;
  const int32_t* n_new;
  const int32_t* group_start;
  const int32_t* prefix_lens;
  PfxWork work;
  unsigned long long wait_ns;
};

struct PfxLaunch {
  CUtensorMap mapK, mapV;  // a layer's planes as [n_pages * n_kv_heads][page][head_dim], boxes of one page
  CUtensorMap mapQ;        // Q as [batch][n_kv_heads][rows][head_dim], boxes of per_tile requests
  CUtensorMap mapQ1;       // the same, boxes of one request
  PfxParams p;
  void* O;
  int grid;
  cudaStream_t stream;
};

// Defined in prefix_attn_d*.cu.
cudaError_t launch_prefix_d64(bool fp16, const PfxLaunch& L);
cudaError_t launch_prefix_d96(bool fp16, const PfxLaunch& L);
cudaError_t launch_prefix_d128(bool fp16, const PfxLaunch& L);

}  // namespace wise
