// Attention of new tokens over a paged cache of 8 or 4 bits.
//
// One block per query row: 128 keys at a time, a thread per key for the logits
// and a thread per channel for the sum of values, with a running maximum and
// sum in fp32.
#include "cache_common.cuh"
#include "quant.cuh"

namespace wise {
namespace {

__device__ float code_value(int bits, const uint8_t* data, int index, uint32_t scale) {
  if (bits == 4) {
    uint32_t h[4];
    q_decode4(data[index >> 1], h);
    const __half2 v = *reinterpret_cast<const __half2*>(&h[0]);
    return __half2float(index & 1 ? __high2half(v) : __low2half(v)) * q_scale_value(scale);
  }
  uint32_t h[2];
  q_decode8(data[index], h);
  return __half2float(__low2half(*reinterpret_cast<const __half2*>(&h[0]))) * q_scale_value(scale);
}

__global__ void __launch_bounds__(128) quant_attn_kernel(const PrefixParams p) {
  __shared__ float q[128], prob[128], part[4];
  __shared__ int pages[128];
  const CacheView& c = p.cache;
  const int D = p.head_dim, tid = threadIdx.x;
  const long long row = blockIdx.x;  // of [batch][n_heads][q_len]
  const int i = (int)(row % p.q_len);
  const int h = (int)(row / p.q_len % p.n_heads), b = (int)(row / p.q_len / p.n_heads);
  const int head = h / p.group;
  const int s = p.slots[b], add = p.n_new ? p.n_new[b] : p.q_len;
  int len = 0;
  if (s >= 0) {
    len = s < c.n_slots ? c.lens[s] : -1;
    if (len < 0 || len > c.max_len || add < 0 || add > p.q_len) {
      if (tid == 0) fault(c, kStatusBadCache);
      len = 0;
    }
  }
  if (row == 0)  // groups are hints that this kernel has no use for, but they are looked at
    for (int g = tid; g < p.n_groups; g += 128)
      if (p.group_start[g] < 0 || p.group_start[g + 1] > p.batch || p.group_start[g] > p.group_start[g + 1])
        fault(c, kStatusBadCache);
  const int e = i < add ? len - add + i + 1 : 0;
  if (p.fp16)
    q[tid] = tid < D ? __half2float(reinterpret_cast<const __half*>(p.Q)[row * D + tid]) : 0.0f;
  else
    q[tid] = tid < D ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.Q)[row * D + tid]) : 0.0f;
  // The whole request gives 0 where it reads a page id out of range.
  int bad = 0;
  if (e > 0)
    for (int k = tid; k < pages_of(c, len); k += 128) bad |= !valid_page(c, c.table[(size_t)s * c.max_pages + k]);
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) fault(c, kStatusBadCache);
  const int T = q_value_tokens(c.bits, c.page);
  const int key_scales = q_key_scales_at(c.bits, D, c.page), values = q_values_at(c.bits, D, c.page),
            value_scales = q_value_scales_at(c.bits, D, c.page), sb = q_key_scale_bytes(D);
  const uint8_t* plane = c.pool + p.layer * c.plane_bytes;
  float m = -INFINITY, l = 0.0f, o = 0.0f;
  for (int k0 = 0; !bad && k0 < e; k0 += 128) {
    const int n = min(128, e - k0);
    float x = -INFINITY;
    if (tid < n) {
      const int page = c.table[(size_t)s * c.max_pages + ((k0 + tid) >> c.page_shift)];
      const int off = (k0 + tid) & (c.page - 1);
      pages[tid] = page;
      const uint8_t* block = plane + (size_t)page * c.page_bytes + (size_t)head * c.head_bytes;
      const int per = 128 / c.bits;  // values of 16 bytes
      x = 0.0f;
      for (int d = 0; d < D; ++d)
        x += q[d] * code_value(c.bits, block + ((size_t)(d / per) * c.page + off) * 16, d % per,
                               block[key_scales + off * sb + d / 16]);
      x *= p.scale_log2;
    }
    float top = x;
    for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    if ((tid & 31) == 0) part[tid >> 5] = top;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    prob[tid] = exp2f(x - m_new);
    __syncthreads();
    const float f = exp2f(m - m_new);
    l *= f;
    o *= f;
    m = m_new;
    for (int j = 0; j < n; ++j) {
      l += prob[j];
      if (tid >= D) continue;
      const uint8_t* block = plane + (size_t)pages[j] * c.page_bytes + (size_t)head * c.head_bytes;
      const int off = (k0 + j) & (c.page - 1);
      o += prob[j] * code_value(c.bits, block + values + ((size_t)(off / T) * D + tid) * (T * c.bits / 8), off % T,
                                block[value_scales + (tid / 16) * c.page + off]);
    }
    __syncthreads();
  }
  if (tid >= D) return;
  const float out = l > 0.0f ? o / l : 0.0f;
  if (p.fp16)
    reinterpret_cast<__half*>(p.O)[row * D + tid] = __float2half_rn(out);
  else
    reinterpret_cast<__nv_bfloat16*>(p.O)[row * D + tid] = __float2bfloat16_rn(out);
}

}  // namespace

size_t quant_attn_workspace(const PrefixParams&, int) { return 0; }

int launch_quant_attn(const PrefixParams& p, void*, int, cudaStream_t stream) {
  quant_attn_kernel<<<(unsigned)(p.batch * p.n_heads * p.q_len), 128, 0, stream>>>(p);
  return cudaGetLastError() == cudaSuccess ? WISE_OK : WISE_ERR_CUDA;
}

}  // namespace wise
