// Attention of new tokens over a paged cache of 8 or 4 bits (wise_kvq_attn):
// the plan, the workspace and the launch.
//
// Mathematics and joining of parts: as in prefix_attn.cuh, with fp16 operands
// (what the cache holds is exact in fp16, see quant.cuh) and fp32 sums.
//
// Work.  With R = q_len * n_heads / n_kv_heads query rows a request and kv head
// there are two kinds of items, each for one kv head, at most 64 rows and a
// range of keys that is taken 128 or 256 at a time (a tile):
//   prefix  the shared prefix of a group against floor(64 / R) of its requests
//           (no sharing where that is 1);
//   own     one request's keys past the shared prefix, its rows 64 at a time.
// The tiles of the own items form one line, those of the prefix items another;
// each is cut into equal runs, one a CTA.  A (run, item) overlap is a segment.
// A segment that is all there is to its rows writes O; the others leave a
// partial result in the workspace slot item + run, unique because both only
// grow along the line, and a second kernel joins them in a fixed order.
#pragma once

#include "prefix_attn.cuh"

namespace wise {

constexpr int kQaRows = 64;

struct QaTotals {
  PfxCuts own, pre;
  int pad[2];
};

struct QaPlan {
  QaTotals* t;
  // Per request.
  int *slot, *len, *lo, *add, *group;
  int* cum;  // [batch + 1] own tiles (of one kv head and row chunk) before it
  // Per group.
  int *start, *lead, *tiles, *row_tiles;
  int* base;  // [n_groups + 1] prefix tiles before it
  int* item;  // [n_groups + 1] prefix items of one kv head before it
};

__host__ __device__ inline int qa_plan_ints(int batch, int n_groups) { return 8 + 6 * batch + 1 + 6 * n_groups + 3; }

__host__ __device__ inline QaPlan qa_plan(int* at, int batch, int n_groups) {
  QaPlan p;
  p.t = reinterpret_cast<QaTotals*>(at);
  p.slot = at + 8;
  p.len = p.slot + batch;
  p.lo = p.len + batch;
  p.add = p.lo + batch;
  p.group = p.add + batch;
  p.cum = p.group + batch;
  p.start = p.cum + batch + 1;
  p.lead = p.start + n_groups + 1;
  p.tiles = p.lead + n_groups;
  p.row_tiles = p.tiles + n_groups;
  p.base = p.row_tiles + n_groups;
  p.item = p.base + n_groups + 1;
  return p;
}

// Workspace: where the merge finds its parts (two int4 per request, kv head
// and row chunk), then for own and prefix segments (m, l) and O as
// [segment][rows] and [segment][rows][head_dim].
struct QaWork {
  int4* sources;
  float2* ml[2];
  float* O[2];
  size_t bytes;
};

inline QaWork qa_work(void* base, int batch, int n_groups, int n_kv_heads, int rows, int head_dim, int sm_count) {
  QaWork w;
  const int chunks = (rows + kQaRows - 1) / kQaRows, per_tile = kQaRows / rows;
  const long long units = (long long)batch * n_kv_heads * chunks;
  const bool shared = n_groups > 0 && per_tile >= 2;
  // A group of m requests has at most m / per_tile + 1 items of a kv head.
  const long long slots[2] = {units + sm_count,
                              shared ? ((long long)batch / per_tile + n_groups) * n_kv_heads + sm_count : 0};
  const int slot_rows[2] = {rows < kQaRows ? rows : kQaRows, kQaRows};
  uint8_t* at = reinterpret_cast<uint8_t*>(base);
  size_t off = 0;
  auto take = [&](size_t n) {
    uint8_t* p = at + off;
    off += (n + 255) / 256 * 256;
    return p;
  };
  w.sources = reinterpret_cast<int4*>(take((size_t)units * 2 * sizeof(int4)));
  for (int k = 0; k < 2; ++k)
    w.ml[k] = reinterpret_cast<float2*>(take((size_t)slots[k] * slot_rows[k] * sizeof(float2)));
  for (int k = 0; k < 2; ++k) w.O[k] = reinterpret_cast<float*>(take((size_t)slots[k] * slot_rows[k] * head_dim * 4));
  w.bytes = off;
  return w;
}

struct QaParams {
  CacheView cache;
  const uint8_t* plane;  // of the layer
  int batch, q_len, n_groups;
  int rows;      // of a request and kv head
  int rows_inv, q_len_inv;  // 65536 / x + 1: n / x = n * that >> 16 for n <= 128, as 128 / 65536 < 1 / x
  int chunks;    // of up to 64 rows
  int keys;      // of a step
  int per_tile;  // requests of a prefix item, 0 where nothing is shared
  int fp16;
  float scale_log2;
  const void* Q;
  void* O;
  const int32_t* slots;
  const int32_t* n_new;
  const int32_t* group_start;
  const int32_t* prefix_lens;
  QaWork work;
  unsigned long long wait_ns;
};

struct QaLaunch {
  QaParams p;
  int grid;
  bool wide;  // items of more than 16 rows
  cudaStream_t stream;
};

// Defined in quant_attn_d*.cu.
cudaError_t launch_quant_attn_d64(const QaLaunch& L);
cudaError_t launch_quant_attn_d96(const QaLaunch& L);
cudaError_t launch_quant_attn_d128(const QaLaunch& L);

}  // namespace wise
