// The quantised paged cache (dtypes WISE_E4M3 and WISE_E2M1 of wise_cache_t):
// the layout of a page and the conversions of a group of 16 values.
//
// Values.  16 neighbouring values of a (token, kv head) row share a scale s, a
// byte read as a number without sign of 5 exponent and 3 mantissa bits: the
// upper bits of the fp16 number, so that s is the byte shifted by 7.  With a =
// the largest size in the group:
//   e2m1 (4 bits)  s = a / 6 rounded to nearest (even), at most 10240;
//                  q = x / s rounded to nearest (even) among 0, 0.5, 1, 1.5, 2,
//                  3, 4, 6 with a sign; 0 where s = 0;
//   e4m3 (8 bits)  s = 2^k, k the smallest in [-15, 7] with a <= 448 * 2^k;
//                  q = x / s rounded to nearest (even), at most 448.
// Every product s q has at most 6 significant bits and lies between 2^-24 and
// 61440, so it is a number of fp16 and of bf16: reading back is exact, and the
// attention multiplies in fp16 whatever type K and V came in.
//
// Layout of the block of one page and kv head (keys and values of `page`
// tokens; blocks are contiguous, so that one bulk copy fetches them):
//   keys          [D * bits / 128][page][16 bytes]   a token's values, 16 bytes at a time
//   key scales    [page][8 bytes] (4 with D = 64)    a token's scales
//   values        [page / T][D][T * bits / 8 bytes]  a channel's values of T tokens, T = 32 (4 bits; 16
//                                                    in pages of 16) or 16 (8 bits)
//   value scales  [D / 16][page]
// So a thread that owns a key (a row of K) or a channel (a row of V^T) reads
// 16 bytes at a time next to its neighbours'.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "internal.cuh"

namespace wise {

__host__ __device__ constexpr int q_key_scale_bytes(int head_dim) { return head_dim == 64 ? 4 : 8; }
__host__ __device__ constexpr int q_value_tokens(int bits, int page) {
  return bits == 8 ? 16 : page < 32 ? 16 : 32;
}
__host__ __device__ constexpr int q_data_bytes(int bits, int head_dim, int page) { return page * head_dim * bits / 8; }
// Offsets in a block.
__host__ __device__ constexpr int q_key_scales_at(int bits, int head_dim, int page) {
  return q_data_bytes(bits, head_dim, page);
}
__host__ __device__ constexpr int q_values_at(int bits, int head_dim, int page) {
  return q_key_scales_at(bits, head_dim, page) + page * q_key_scale_bytes(head_dim);
}
__host__ __device__ constexpr int q_value_scales_at(int bits, int head_dim, int page) {
  return q_values_at(bits, head_dim, page) + q_data_bytes(bits, head_dim, page);
}
__host__ __device__ constexpr int q_block_bytes(int bits, int head_dim, int page) {
  return q_value_scales_at(bits, head_dim, page) + page * (head_dim / 16);
}

#ifdef __CUDACC__

// The scale of a group as its byte, from the group's largest size.
__device__ __forceinline__ uint32_t q_scale4(float a) {
  const float t = __fdiv_rn(a, 6.0f);  // exact ties of a / 6 stay ties: a has at most 11 significant bits
  if (t >= 10240.0f) return 28 * 8 + 2;
  if (t < 6.103515625e-05f) return (uint32_t)__float2int_rn(t * 131072.0f);  // below 2^-14: steps of 2^-17
  uint32_t u = __float_as_uint(t);
  u += 0x7FFFFu + ((u >> 20) & 1u);
  return (u >> 20) - (112u << 3);
}
__device__ __forceinline__ uint32_t q_scale8(float a) {
  int k = (int)((__float_as_uint(a) + 0x1FFFFFu) >> 23) - 127 - 8;  // a <= 1.75 * 2^(k + 8)
  k = min(max(k, -15), 7);
  return k == -15 ? 4u : (uint32_t)(k + 15) << 3;
}
__device__ __forceinline__ float q_scale_value(uint32_t byte) {
  return __half2float(__ushort_as_half((unsigned short)(byte << 7)));
}

// Eight values to one word of e2m1, the first in the lowest bits; inv is 1 / s
// rounded up.  A quotient x / s that lies half way between two codes is then
// hit exactly by x * inv rounded towards zero (the product exceeds it by less
// than a unit in the last place); other quotients differ from those points by
// more than 2^-12 (x has at most 11 significant bits, a point half way times s
// at most 7).
__device__ __forceinline__ uint32_t q_codes4(const float (&x)[8], float inv) {
  uint32_t w;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __fmul_rz(x[i], inv);
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return w;
}
// Four values to one word of e4m3 (1 / s is a power of two, so x / s is exact).
__device__ __forceinline__ uint32_t q_codes8(float x0, float x1, float x2, float x3, float inv) {
  uint32_t w;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
      "mov.b32 %0, {a, b};\n\t}"
      : "=r"(w)
      : "f"(x0 * inv), "f"(x1 * inv), "f"(x2 * inv), "f"(x3 * inv));
  return w;
}

// A word of codes to fp16 pairs, before the scale.
__device__ __forceinline__ void q_decode4(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
__device__ __forceinline__ void q_decode8(uint32_t w, uint32_t (&h)[2]) {
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(h[0]), "=r"(h[1])
      : "r"(w));
}
__device__ __forceinline__ uint32_t q_mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

#endif  // __CUDACC__

}  // namespace wise
