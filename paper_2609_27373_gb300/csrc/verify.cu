// Verification of drafted tokens against the target's probabilities, from
// given random numbers (the rule stands in include/wise.h).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <limits.h>

#include "internal.cuh"

namespace wise {
namespace {

constexpr int kThreads = 1024;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

// Fixed-point weight floor(min(x, 1) * 2^40); the product by a power of two is
// exact, and NaN and negative values give 0.
__device__ __forceinline__ unsigned long long weight(float x) {
  return x > 0.0f ? (unsigned long long)(fminf(x, 1.0f) * 1099511627776.0f) : 0ull;
}

__device__ __forceinline__ unsigned long long warp_inclusive(unsigned long long v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyParams a) {
  __shared__ unsigned long long sums[kThreads / 32];
  __shared__ int first_refusal, bad_token, found;
  const int b = blockIdx.x, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const T* p = reinterpret_cast<const T*>(a.p) + (size_t)b * (a.k_max + 1) * a.vocab;
  const T* q = reinterpret_cast<const T*>(a.q) + (size_t)b * a.k_max * a.vocab;
  int n_draft = a.n_draft ? a.n_draft[b] : a.k_max;
  if (n_draft < 0 || n_draft > a.k_max) {
    if (threadIdx.x == 0) atomicOr(a.status, kStatusBadCache);
    n_draft = n_draft < 0 ? 0 : a.k_max;
  }
  if (threadIdx.x == 0) {
    first_refusal = n_draft;
    bad_token = INT_MAX;
    found = -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_draft; i += kThreads) {
    const int x = a.draft[(size_t)b * a.k_max + i];
    bool stands = false;
    if (x < 0 || x >= a.vocab) {
      atomicMin(&bad_token, i);
    } else {
      const float px = to_f32(p[(size_t)i * a.vocab + x]), qx = to_f32(q[(size_t)i * a.vocab + x]);
      stands = __fmul_rn(a.u_accept[(size_t)b * a.k_max + i], qx) < px;
    }
    if (!stands) atomicMin(&first_refusal, i);
  }
  __syncthreads();
  const int n = first_refusal;
  const bool use_p = n == n_draft || bad_token == n;
  if (threadIdx.x == 0 && bad_token <= n && n < n_draft) atomicOr(a.status, kStatusBadCache);
  const T* prow = p + (size_t)n * a.vocab;
  const T* qrow = q + (size_t)n * a.vocab;
  // Each warp owns a contiguous part of the vocabulary.
  const int part = (a.vocab + kThreads / 32 - 1) / (kThreads / 32);
  const int v0 = min(w * part, a.vocab), v1 = min(v0 + part, a.vocab);
  unsigned long long total = 0, before = 0;
  bool residual = !use_p;
  auto at = [&](int v) -> unsigned long long {
    const float pv = to_f32(prow[v]);
    return weight(residual ? pv - to_f32(qrow[v]) : pv);
  };
  for (;;) {
    unsigned long long mine = 0;
    for (int v = v0 + lane; v < v1; v += 32) mine += at(v);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) sums[w] = mine;
    __syncthreads();
    total = 0;
    before = 0;
    for (int k = 0; k < kThreads / 32; ++k) {
      if (k < w) before += sums[k];
      total += sums[k];
    }
    __syncthreads();
    if (total > 0 || !residual) break;
    residual = false;  // p <= q everywhere: the target row itself
  }
  const float us = a.u_sample[b];
  const unsigned long long u = (unsigned long long)(fminf(fmaxf(us, 0.0f), 1.0f - 0x1p-24f) * 16777216.0f);
  // floor(total * u / 2^24) without leaving 64 bits.
  const unsigned long long t = (total >> 24) * u + (((total & 0xFFFFFFull) * u) >> 24);
  if (total > 0 && before <= t) {
    unsigned long long run = before;
    for (int c0 = v0; c0 < v1; c0 += 32) {
      const int v = c0 + lane;
      const unsigned long long upto = run + warp_inclusive(v < v1 ? at(v) : 0ull, lane);
      const unsigned hit = __ballot_sync(0xffffffffu, v < v1 && upto > t);
      if (hit) {
        if (lane == __ffs(hit) - 1) found = v;
        break;
      }
      run = __shfl_sync(0xffffffffu, upto, 31);
    }
  }
  // Only the warp whose part holds the crossing finds it: an earlier part ends
  // at or below t.  Later parts start above t and do not look.
  __syncthreads();
  for (int i = threadIdx.x; i <= a.k_max; i += kThreads)
    a.tokens[(size_t)b * (a.k_max + 1) + i] = i < n ? a.draft[(size_t)b * a.k_max + i] : i == n ? found : -1;
  if (threadIdx.x == 0) a.accepted[b] = n;
}

}  // namespace

cudaError_t launch_verify_draft(int dtype, const VerifyParams& p, cudaStream_t stream) {
  if (dtype == WISE_BF16)
    verify_kernel<__nv_bfloat16><<<p.batch, kThreads, 0, stream>>>(p);
  else if (dtype == WISE_FP16)
    verify_kernel<__half><<<p.batch, kThreads, 0, stream>>>(p);
  else
    verify_kernel<float><<<p.batch, kThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace wise
