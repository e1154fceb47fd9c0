// Attention of new tokens over the paged cache (wise_prefix_attn): one block
// per query row, online softmax over tiles of 128 keys in fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_common.cuh"
#include "internal.cuh"

namespace wise {
namespace {

constexpr int kKeys = 128;

__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f32(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_f32(__half& y, float x) { y = __float2half_rn(x); }

template <int D, typename T>
__global__ void __launch_bounds__(kKeys) row_attn_kernel(const PrefixParams p) {
  __shared__ float q[D], w[kKeys], red[4];
  __shared__ int page_of[8];
  const CacheView& c = p.cache;
  const int i = blockIdx.x % p.q_len;
  const int bh = blockIdx.x / p.q_len;
  const int h = bh % p.n_heads, b = bh / p.n_heads, kvh = h / p.group;
  const int t = threadIdx.x, lane = t & 31, wq = t >> 5;
  const size_t row = ((size_t)bh * p.q_len + i) * D;
  const int s = p.slots[b];
  int seen = 0;
  if (s >= c.n_slots) {
    if (t == 0) atomicOr(c.status, kStatusBadCache);
  } else if (s >= 0) {
    const int len = c.lens[s], add = p.n_new ? p.n_new[b] : p.q_len;
    if (len < 0 || len > c.max_len || add < 0 || add > p.q_len) {
      if (t == 0) atomicOr(c.status, kStatusBadCache);
    } else if (i < add) {
      seen = max(0, len - add + i + 1);
    }
  }
  if (blockIdx.x == 0) {
    for (int g = t; g < p.n_groups; g += kKeys) {
      const int a = p.group_start[g], e = p.group_start[g + 1];
      if (a < 0 || a > e || e > p.batch) atomicOr(c.status, kStatusBadCache);
    }
  }
  if (t < D) q[t] = to_f32(reinterpret_cast<const T*>(p.Q)[row + t]) * p.scale_log2;
  float m = -INFINITY, l = 0.0f, acc = 0.0f;
  const uint8_t* kplane = c.pool + (2 * p.layer) * c.plane_bytes + (size_t)kvh * c.head_bytes;
  const uint8_t* vplane = kplane + c.plane_bytes;
  for (int k0 = 0; k0 < seen; k0 += kKeys) {
    __syncthreads();
    if (t < kKeys / c.page) {
      const int at = k0 / c.page + t;
      int page = at < c.max_pages && at * c.page < seen ? c.table[(size_t)s * c.max_pages + at] : -1;
      if (at * c.page < seen && (page < 0 || page >= c.n_pages)) {
        atomicOr(c.status, kStatusBadCache);
        page = -1;
      }
      page_of[t] = page;
    }
    __syncthreads();
    float x = -INFINITY;
    if (k0 + t < seen) {
      const int page = page_of[t / c.page];
      x = 0.0f;
      if (page >= 0) {
        const T* k = reinterpret_cast<const T*>(kplane + (size_t)page * c.page_bytes) + (size_t)(t % c.page) * D;
        for (int d = 0; d < D; ++d) x += q[d] * to_f32(k[d]);
      }
    }
    float tile_max = x;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) tile_max = fmaxf(tile_max, __shfl_xor_sync(0xffffffffu, tile_max, o));
    if (lane == 0) red[wq] = tile_max;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float f = ex2_approx(m - m_new);
    m = m_new;
    w[t] = k0 + t < seen ? ex2_approx(x - m) : 0.0f;
    __syncthreads();
    acc *= f;
    l *= f;
    for (int j = 0; j < min(kKeys, seen - k0); ++j) {
      l += w[j];
      const int page = page_of[j / c.page];
      if (t < D && page >= 0)
        acc += w[j] * to_f32(reinterpret_cast<const T*>(vplane + (size_t)page * c.page_bytes)[(size_t)(j % c.page) * D + t]);
    }
  }
  if (t < D) from_f32(reinterpret_cast<T*>(p.O)[row + t], l > 0.0f ? acc / l : 0.0f);
}

template <int D>
cudaError_t launch(const PrefixParams& p, cudaStream_t stream) {
  const int grid = p.batch * p.n_heads * p.q_len;
  if (p.fp16)
    row_attn_kernel<D, __half><<<grid, kKeys, 0, stream>>>(p);
  else
    row_attn_kernel<D, __nv_bfloat16><<<grid, kKeys, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

size_t prefix_attn_workspace(const PrefixParams&, int) { return 0; }

cudaError_t launch_prefix_attn(const PrefixParams& p, void*, int, cudaStream_t stream) {
  switch (p.head_dim) {
    case 64: return launch<64>(p, stream);
    case 96: return launch<96>(p, stream);
    default: return launch<128>(p, stream);
  }
}

}  // namespace wise
