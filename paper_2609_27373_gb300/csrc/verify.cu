// Verification of drafted tokens against the target's probabilities, from
// given random numbers (the rule stands in include/wise.h).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <limits.h>

#include "internal.cuh"

namespace wise {
namespace {

namespace cg = cooperative_groups;

// A request is one cluster of 1, 2, 4 or 8 blocks, each with a contiguous
// slice of the vocabulary and each of its warps with a contiguous part of
// that.  The rows of probabilities are read once: every block finds the first
// refusal by itself (two dependent loads), the warps add up their parts'
// weights, the blocks exchange their sums through distributed shared memory,
// and the block that holds the crossing reads the crossing part (at most 8192
// tokens, by now in L2) once more, a few tokens per thread.  What bounds it:
// memory for full batches, at less than its bandwidth since blocks with one row
// run beside blocks with two and their set-up beside nothing (160 x 131075 tokens
// in fp32, one wave: 34 us, 4.1 TB/s; 320: 56 us, 5.0 TB/s), the chain of
// dependent loads and the cluster barrier for a few requests (5.1 us).  Blocks of 256 threads, five an SM, keep
// requests in different phases side by side (512 threads, two an SM: 45 us for
// the 160).
constexpr int kThreads = 256;
constexpr int kBlocksPerSM = 5;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

// The fixed-point weight floor(min(x, 1) * 2^40) of x >= 0 (NaN counts as 0) in
// two parts, hi * 2^23 + lo, by additions that round toward zero: x + 64 keeps
// the multiples of 2^-17 of x in its significand, the rest of x (exact) scaled
// by 2^17 and added to 1 keeps 23 more bits.  Sums of the bit patterns minus
// their constant parts are sums of hi and lo.  (A conversion to 64-bit
// integers goes through the FP64 pipe, which then bounds the kernel: 160 rows
// of 131075 tokens in fp32 took 70 us that way, 57 us with 64-bit shifts.)
struct Weight {
  uint32_t hi, lo;  // bit patterns, kHiZero + hi and kLoZero + lo
};
constexpr uint32_t kHiZero = 0x42800000u;  // 64.0f
constexpr uint32_t kLoZero = 0x3F800000u;  // 1.0f
__device__ __forceinline__ Weight weight_bits(float x) {
  const float y = __saturatef(x);
  const float a = __fadd_rz(y, 64.0f);
  const float rest = y - (a - 64.0f);
  return Weight{__float_as_uint(a), __float_as_uint(__fmaf_rz(rest, 131072.0f, 1.0f))};
}
__device__ __forceinline__ unsigned long long weight(float x) {
  const Weight w = weight_bits(x);
  return ((unsigned long long)(w.hi - kHiZero) << 23) + (w.lo - kLoZero);
}

// Inclusive prefix sum over the block of one value per thread.
__device__ __forceinline__ unsigned long long block_inclusive(unsigned long long v, unsigned long long* sums) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  if (lane == 31) sums[w] = v;
  __syncthreads();
  for (int k = 0; k < w; ++k) v += sums[k];
  return v;
}

// The weights' sum over tokens v0 .. v1 - 1 of a row, per lane.  VEC tokens
// are loaded at a time (16 bytes when the rows allow it, else one), kBatch
// loads of each row in flight.  A lane adds up at most 2^18 / (4 * kThreads)
// = 256 weights (vocabularies past 2^12 take at least 4 blocks), so that the parts' sums fit 32 bits.
template <typename T, int VEC, bool RESIDUAL>
__device__ __forceinline__ unsigned long long part_sum(const T* p, const T* q, int v0, int v1, int lane) {
  struct alignas(sizeof(T) * VEC) Pack {
    T x[VEC];
  };
  constexpr int kBatch = VEC == 1 ? 8 : VEC == 4 ? 4 : 2;
  constexpr int kStep = 32 * VEC;
  uint32_t hi = 0, lo = 0, count = 0;
  auto add = [&](const Pack& a, const Pack& b) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const Weight w = weight_bits(RESIDUAL ? to_f32(a.x[e]) - to_f32(b.x[e]) : to_f32(a.x[e]));
      hi += w.hi;
      lo += w.lo;
    }
    count += VEC;
  };
  int v = v0 + lane * VEC;
  for (; v + (kBatch - 1) * kStep < v1; v += kBatch * kStep) {
    Pack a[kBatch], b[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      a[k] = *reinterpret_cast<const Pack*>(p + v + k * kStep);
      if (RESIDUAL) b[k] = *reinterpret_cast<const Pack*>(q + v + k * kStep);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) add(a[k], b[k]);
  }
  for (; v < v1; v += kStep) {
    Pack a, b;
    a = *reinterpret_cast<const Pack*>(p + v);
    if (RESIDUAL) b = *reinterpret_cast<const Pack*>(q + v);
    add(a, b);
  }
  return ((unsigned long long)(hi - count * kHiZero) << 23) + (lo - count * kLoZero);
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads, kBlocksPerSM) verify_kernel(const VerifyParams a) {
  __shared__ unsigned long long sums[kWarps], scan_sums[kWarps];
  __shared__ unsigned long long block_sum[2];
  __shared__ int first_refusal, bad_token;
  const cg::cluster_group cluster = cg::this_cluster();
  const int n_blocks = cluster.num_blocks(), rank = cluster.block_rank();
  const int b = blockIdx.x / n_blocks, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const T* p = reinterpret_cast<const T*>(a.p) + (size_t)b * (a.k_max + 1) * a.vocab;
  const T* q = reinterpret_cast<const T*>(a.q) + (size_t)b * a.k_max * a.vocab;
  int n_draft = a.n_draft ? a.n_draft[b] : a.k_max;
  if (n_draft < 0 || n_draft > a.k_max) {
    if (rank == 0 && threadIdx.x == 0) atomicOr(a.status, kStatusBadCache);
    n_draft = n_draft < 0 ? 0 : a.k_max;
  }
  if (threadIdx.x == 0) {
    first_refusal = n_draft;
    bad_token = INT_MAX;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.k_max; i += kThreads) {
    const int x = a.draft[(size_t)b * a.k_max + i];
    const float u = a.u_accept[(size_t)b * a.k_max + i];
    bool stands = false;
    if (x >= 0 && x < a.vocab) {
      const float px = to_f32(p[(size_t)i * a.vocab + x]), qx = to_f32(q[(size_t)i * a.vocab + x]);
      stands = __fmul_rn(u, qx) < px;
    } else if (i < n_draft) {
      atomicMin(&bad_token, i);
    }
    if (!stands && i < n_draft) atomicMin(&first_refusal, i);
  }
  const float us = a.u_sample[b];
  __syncthreads();
  const int n = first_refusal;
  bool residual = n < n_draft && bad_token != n;
  if (rank == 0 && threadIdx.x == 0 && bad_token == n) atomicOr(a.status, kStatusBadCache);
  const T* prow = p + (size_t)n * a.vocab;
  const T* qrow = q + (size_t)n * a.vocab;
  const int part = ((a.vocab + n_blocks * kWarps - 1) / (n_blocks * kWarps) + VEC - 1) / VEC * VEC;
  const int first = rank * kWarps * part;  // of the block
  const int v0 = min(first + w * part, a.vocab), v1 = min(v0 + part, a.vocab);
  unsigned long long total = 0, before = 0;
  for (int round = 0;; ++round) {
    unsigned long long mine = residual ? part_sum<T, VEC, true>(prow, qrow, v0, v1, lane)
                                       : part_sum<T, VEC, false>(prow, qrow, v0, v1, lane);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) sums[w] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
      unsigned long long s = 0;
      for (int k = 0; k < kWarps; ++k) s += sums[k];
      block_sum[round] = s;
    }
    cluster.sync();
    total = 0;
    before = 0;
    for (int k = 0; k < n_blocks; ++k) {
      const unsigned long long s = *cluster.map_shared_rank(&block_sum[round], k);
      if (k < rank) before += s;
      total += s;
    }
    if (total > 0 || !residual) break;
    residual = false;  // p <= q everywhere: the target row itself
    __syncthreads();
  }
  // The other blocks' sums have been read; a block may exit once all have.
  asm volatile("barrier.cluster.arrive;" ::: "memory");
  const unsigned long long u = (unsigned long long)(fminf(fmaxf(us, 0.0f), 1.0f - 0x1p-24f) * 16777216.0f);
  // floor(total * u / 2^24) without leaving 64 bits; below total.
  const unsigned long long t = (total >> 24) * u + (((total & 0xFFFFFFull) * u) >> 24);
  int32_t* tokens = a.tokens + (size_t)b * (a.k_max + 1);
  unsigned long long mine = 0;
  for (int k = 0; k < kWarps; ++k) mine += sums[k];
  if (total > 0 && before <= t && t < before + mine) {
    // The crossing lies in this block: its part, then its token.
    int c = 0;
    while (before + sums[c] <= t) before += sums[c++];
    const int c0 = min(first + c * part, a.vocab), c1 = min(c0 + part, a.vocab);
    const int each = (part + kThreads - 1) / kThreads;
    const int e0 = min(c0 + (int)threadIdx.x * each, c1), e1 = min(e0 + each, c1);
    auto at = [&](int v) {
      const float pv = to_f32(prow[v]);
      return weight(residual ? pv - to_f32(qrow[v]) : pv);
    };
    unsigned long long s = 0;
    for (int v = e0; v < e1; ++v) s += at(v);
    unsigned long long upto = before + block_inclusive(s, scan_sums);
    if (upto > t && upto - s <= t) {
      upto -= s;
      int v = e0;
      while ((upto += at(v)) <= t) ++v;
      tokens[n] = v;
    }
  } else if (total == 0 && rank == 0 && threadIdx.x == 0) {
    tokens[n] = -1;
  }
  if (rank == 0) {
    for (int i = threadIdx.x; i <= a.k_max; i += kThreads)
      if (i != n) tokens[i] = i < n ? a.draft[(size_t)b * a.k_max + i] : -1;
    if (threadIdx.x == 0) a.accepted[b] = n;
  }
  asm volatile("barrier.cluster.wait;" ::: "memory");
}

template <typename T, int VEC>
cudaError_t launch_instance(const VerifyParams& p, cudaStream_t stream) {
  // Blocks of a request: fewer for small vocabularies, where 8 would have
  // little to read each, and 4 once 8 a request are more than one wave (320
  // requests of 65536 in bf16: 21.8 us with 4, 28.8 with 8; 80, one wave: 8.4
  // and 8.5; 40 of 131075 in fp32: 18.0 and 12.6).
  int cluster = (long long)p.batch * 8 > (long long)p.sm_count * kBlocksPerSM ? 4 : 8;
  while (cluster > 1 && p.vocab <= cluster * kThreads * 4) cluster /= 2;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.batch * cluster);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, verify_kernel<T, VEC>, p);
}

template <typename T>
cudaError_t launch_type(const VerifyParams& p, cudaStream_t stream) {
  constexpr int kVec = 16 / sizeof(T);
  const bool aligned = p.vocab % kVec == 0 && reinterpret_cast<uintptr_t>(p.p) % 16 == 0 &&
                       reinterpret_cast<uintptr_t>(p.q) % 16 == 0;
  return aligned ? launch_instance<T, kVec>(p, stream) : launch_instance<T, 1>(p, stream);
}

}  // namespace

cudaError_t launch_verify_draft(int dtype, const VerifyParams& p, cudaStream_t stream) {
  if (dtype == WISE_BF16)
    return launch_type<__nv_bfloat16>(p, stream);
  if (dtype == WISE_FP16)
    return launch_type<__half>(p, stream);
  return launch_type<float>(p, stream);
}

}  // namespace wise
