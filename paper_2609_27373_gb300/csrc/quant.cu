// Storing keys and values in a paged cache of 8 or 4 bits, and reading rows of
// any cache back.  Formulas and layout: quant.cuh.
//
// A warp takes 32 neighbouring positions of a sequence (a span, aligned to 32)
// of one kv head, of the keys or of the values (blockIdx.y), and goes through
// their channels 32 at a time; where that gives too few warps, each takes 32
// channels.  Outside the cache a lane is a token: it reads or writes 64
// neighbouring bytes of that token's row, two groups with a scale each.  In the
// cache that holds for keys too; values lie by channels, so a warp transposes
// its 32 x 32 codes in registers, exchanging lane bit i with index bit i at a
// time.
//
// 2 x 32K tokens of 8 heads of 128 are stored in 4 bits in 65 us (343 MB read and
// written, 5.3 of a copy's 6.8 TB/s) and read back in 66.  Storing is bound by
// latency: with 64 registers a thread half of the warps that an SM holds are there,
// and they take 63 of 100 issue slots (16 values need their maximum, a quotient, a
// reciprocal and 16 products and roundings) and 56 of DRAM's, a third of their time
// waiting for K and V.  Reading is next to what L1 takes, 86 of 100 of its cycles
// (41 of the issue slots, 51 of DRAM's): the lanes of a warp write 32 bytes of a row
// each; in 8 bits 64 of 100, and latency.  With a warp for 32 channels of a span at
// any size storing and reading back took 199 us together and reading 103.
#include <algorithm>

#include "cache_common.cuh"
#include "quant.cuh"

namespace wise {
namespace {

constexpr int kIoThreads = 256;
constexpr int kIoWarps = kIoThreads / 32;

// Offsets in a block.
struct QuantShape {
  int key_scales, values, value_scales, key_scale_bytes;
};

// 32 x 32 codes: word w of a lane holds the codes of indexes per * w ...,
// per = 8 (4 bits) or 4 (8 bits); afterwards lane and index are exchanged.
template <int BITS>
__device__ __forceinline__ void transpose_codes(uint32_t (&w)[BITS], int lane) {
#pragma unroll
  for (int b = 16; b * BITS / 32 > 0; b >>= 1) {  // index bits that choose the word
    const int step = b * BITS / 32;
    const bool up = lane & b;
#pragma unroll
    for (int k = 0; k < BITS; ++k) {
      if (k & step) continue;
      const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[k] : w[k + step], b);
      if (up)
        w[k] = got;
      else
        w[k + step] = got;
    }
  }
  if (BITS == 4) {
    const uint32_t pick = lane & 4 ? 0x3276u : 0x5410u;
#pragma unroll
    for (int k = 0; k < BITS; ++k) w[k] = __byte_perm(w[k], __shfl_xor_sync(0xffffffffu, w[k], 4), pick);
  } else {
    const uint32_t pick = lane & 2 ? 0x3276u : 0x5410u;
#pragma unroll
    for (int k = 0; k < BITS; ++k) w[k] = __byte_perm(w[k], __shfl_xor_sync(0xffffffffu, w[k], 2), pick);
  }
  constexpr int kByteBit = BITS == 4 ? 2 : 1;
  const uint32_t pick = lane & kByteBit ? 0x3715u : 0x6240u;
#pragma unroll
  for (int k = 0; k < BITS; ++k) w[k] = __byte_perm(w[k], __shfl_xor_sync(0xffffffffu, w[k], kByteBit), pick);
  if (BITS == 4) {
    const bool up = lane & 1;
    const uint32_t keep = up ? 0xF0F0F0F0u : 0x0F0F0F0Fu;
#pragma unroll
    for (int k = 0; k < BITS; ++k) {
      const uint32_t y = __shfl_xor_sync(0xffffffffu, w[k], 1);
      w[k] = (w[k] & keep) | ((up ? y >> 4 : y << 4) & ~keep);
    }
  }
}

template <bool FP16>
__device__ __forceinline__ float2 widen(uint32_t v) {
  if (FP16) return __half22float2(*reinterpret_cast<const __half2*>(&v));
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// The largest size of 16 values (NaN passed over).
template <bool FP16>
__device__ __forceinline__ float largest(const uint4& a, const uint4& b) {
  const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (FP16) {
    __half2 m = __habs2(*reinterpret_cast<const __half2*>(&v[0]));
#pragma unroll
    for (int k = 1; k < 8; ++k) m = __hmax2(m, __habs2(*reinterpret_cast<const __half2*>(&v[k])));
    const float2 f = __half22float2(m);
    return fmaxf(f.x, f.y);
  }
  __nv_bfloat162 m = __habs2(*reinterpret_cast<const __nv_bfloat162*>(&v[0]));
#pragma unroll
  for (int k = 1; k < 8; ++k) m = __hmax2(m, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&v[k])));
  const float2 f = __bfloat1622float2(m);
  return fmaxf(f.x, f.y);
}

// 16 values to their codes (BITS / 2 words) and the byte of their scale.
template <int BITS, bool FP16>
__device__ __forceinline__ uint32_t encode_group(const uint4& a, const uint4& b, uint32_t* w) {
  float m = largest<FP16>(a, b);
  if (!(m >= 0.0f)) m = 0.0f;  // all NaN
  const uint32_t byte = BITS == 4 ? q_scale4(m) : q_scale8(m);
  const float inv = byte ? __frcp_ru(q_scale_value(byte)) : 0.0f;
  const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int k = 0; k < 8; k += 4) {
    const float2 f0 = widen<FP16>(v[k]), f1 = widen<FP16>(v[k + 1]), f2 = widen<FP16>(v[k + 2]),
                 f3 = widen<FP16>(v[k + 3]);
    if (BITS == 4) {
      const float x[8] = {f0.x, f0.y, f1.x, f1.y, f2.x, f2.y, f3.x, f3.y};
      w[k / 4] = q_codes4(x, inv);
    } else {
      w[k / 2] = q_codes8(f0.x, f0.y, f1.x, f1.y, inv);
      w[k / 2 + 1] = q_codes8(f2.x, f2.y, f3.x, f3.y, inv);
    }
  }
  return byte;
}

// 16 codes to values.
template <int BITS, bool FP16>
__device__ __forceinline__ void decode_group(const uint32_t* w, uint32_t byte, uint32_t (&out)[8]) {
  const uint32_t s = byte << 7 | byte << 23;
  if (BITS == 4) {
    uint32_t h[4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      q_decode4(w[k], h);
#pragma unroll
      for (int j = 0; j < 4; ++j) out[4 * k + j] = q_mul2(h[j], s);
    }
  } else {
    uint32_t h[2];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      q_decode8(w[k], h);
      out[2 * k] = q_mul2(h[0], s);
      out[2 * k + 1] = q_mul2(h[1], s);
    }
  }
  if constexpr (!FP16) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&out[k]));
      const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
      out[k] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
}

// 32-token spans that `rows` neighbouring positions can touch.
__host__ __device__ inline int spans_of(int rows) { return (rows + 30) / 32 + 1; }

// --------------------------------------------------------------------- write
// A warp's share of the values of one chunk of T tokens that lie in one page:
// w[..] holds lane = channel, index = token.  New tokens start at `from` of the
// chunk; those before it stay as they are.
template <int WORDS, int BITS>
__device__ __forceinline__ void store_chunk(uint8_t* to, const uint32_t* w, int from) {
  uint32_t v[WORDS], old[WORDS];
#pragma unroll
  for (int k = 0; k < WORDS; ++k) v[k] = w[k];
  if (from > 0) {
    if constexpr (WORDS == 4)
      *reinterpret_cast<uint4*>(old) = *reinterpret_cast<const uint4*>(to);
    else
      *reinterpret_cast<uint2*>(old) = *reinterpret_cast<const uint2*>(to);
#pragma unroll
    for (int k = 0; k < WORDS; ++k) {
      const int n = min(max(from * BITS - 32 * k, 0), 32);  // bits of the word that stay
      const uint32_t stay = n == 32 ? 0xffffffffu : (1u << n) - 1u;
      v[k] = (old[k] & stay) | (v[k] & ~stay);
    }
  }
  if constexpr (WORDS == 4)
    *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(v);
  else
    *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(v);
}

// Work of one warp: spans of heads, and for each all channels or 32 of them.
struct QuantJobs {
  int parts;    // of 32 channels, of a row
  int per_job;  // of them that a job has: all or 1
  int spans;
  int jobs;
  bool wide;    // K and V are aligned to 32 bytes
};

// 64 bytes of a row.
__device__ __forceinline__ void load_row(const uint8_t* at, bool wide, uint4 (&x)[4]) {
  if (wide) {
#pragma unroll
    for (int k = 0; k < 4; k += 2)
      asm volatile("ld.global.nc.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(x[k].x), "=r"(x[k].y), "=r"(x[k].z), "=r"(x[k].w), "=r"(x[k + 1].x), "=r"(x[k + 1].y),
                     "=r"(x[k + 1].z), "=r"(x[k + 1].w)
                   : "l"(at + 16 * k));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __ldg(reinterpret_cast<const uint4*>(at) + k);
  }
}
__device__ __forceinline__ void store_row(uint8_t* at, bool wide, const uint4 (&x)[4]) {
  if (wide) {
#pragma unroll
    for (int k = 0; k < 4; k += 2)
      asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(x[k].x), "r"(x[k].y), "r"(x[k].z),
                   "r"(x[k].w), "r"(x[k + 1].x), "r"(x[k + 1].y), "r"(x[k + 1].z), "r"(x[k + 1].w), "l"(at + 16 * k)
                   : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(at)[k] = x[k];
  }
}

template <int BITS, bool FP16>
__global__ void __launch_bounds__(kIoThreads, 4) quant_write_kernel(const QuantIo io, const QuantShape sh,
                                                                    const QuantJobs jb) {
  extern __shared__ uint32_t seen[];
  const CacheView& c = io.cache;
  const int lane = threadIdx.x & 31;
  const uint32_t* twice = io.batch > 1 ? mark_twice(c, io.slots, io.batch, seen) : nullptr;
  const bool values = blockIdx.y;
  const uint8_t* in = reinterpret_cast<const uint8_t*>(values ? io.V : io.K);
  uint8_t* plane = c.pool + io.layer * c.plane_bytes;
  for (int job = blockIdx.x * kIoWarps + threadIdx.x / 32; job < jb.jobs; job += gridDim.x * kIoWarps) {
    const int unit = jb.per_job == 1 ? job / jb.parts : job;
    const int part0 = jb.per_job == 1 ? job - unit * jb.parts : 0;
    const int bh = unit / jb.spans, span = unit - bh * jb.spans;
    const int b = bh / c.n_kv_heads, head = bh - b * c.n_kv_heads;
    const int s = io.slots[b], add = io.count ? io.count[b] : io.rows;
    if (s < 0) continue;
    const bool in_range = s < c.n_slots && !(twice && ((twice[s >> 5] >> (s & 31)) & 1u));
    const int len = in_range ? c.lens[s] : -1;
    if (len < 0 || len > c.max_len || add < 0 || add > io.rows || add > len) {
      if (lane == 0) fault(c, kStatusBadCache);
      continue;
    }
    const int start = len - add;
    if (add == 0 || span > (len - 1 - (start & ~31)) / 32) continue;
    const int base = (start & ~31) + 32 * span;
    const int pos = base + lane;
    const bool on = pos >= start && pos < len;
    const uint8_t* row = in + (((size_t)bh * io.rows + (on ? pos - start : 0)) * io.head_dim + 32 * part0) * 2;
    uint4 x[4] = {};
    if (on) load_row(row, jb.wide, x);
    int page = -1;
    if (on) {
      page = c.table[(size_t)s * c.max_pages + (pos >> c.page_shift)];
      if (!valid_page(c, page) || c.refs[page] > 1) {
        fault(c, kStatusBadCache);
        page = -1;
      }
    }
    const int off = pos & (c.page - 1);
    uint8_t* block = plane + (size_t)max(page, 0) * c.page_bytes + (size_t)head * c.head_bytes;
    // The span's pieces of values in the cache: T tokens each, in one page.
    const int T = BITS == 8 || c.page == 16 ? 16 : 32;
    const int from0 = max(start - base, 0), from1 = max(start - (base + 16), 0);  // first new tokens
    const int page0 = __shfl_sync(0xffffffffu, page, min(from0, 31));
    const int page1 = __shfl_sync(0xffffffffu, page, min(16 + from1, 31));
#pragma unroll 1
    for (int part = part0; part < part0 + jb.per_job; ++part) {
      uint32_t w[BITS];
      const uint32_t s0 = encode_group<BITS, FP16>(x[0], x[1], w);
      const uint32_t s1 = encode_group<BITS, FP16>(x[2], x[3], w + BITS / 2);
      if (on && part + 1 < part0 + jb.per_job) {  // the next channels are on their way meanwhile
        row += 64;
        load_row(row, jb.wide, x);
      }
      if (!values) {
        if (page >= 0) {
          uint8_t* to = block + ((size_t)part * (BITS / 4) * c.page + off) * 16;
          *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(w);
          if (BITS == 8) *reinterpret_cast<uint4*>(to + c.page * 16) = *reinterpret_cast<const uint4*>(w + BITS / 2);
          *reinterpret_cast<uint16_t*>(block + sh.key_scales + off * sh.key_scale_bytes + 2 * part) =
              (uint16_t)(s0 | s1 << 8);
        }
        continue;
      }
      if (page >= 0) {
        block[sh.value_scales + 2 * part * c.page + off] = (uint8_t)s0;
        block[sh.value_scales + (2 * part + 1) * c.page + off] = (uint8_t)s1;
      }
      transpose_codes<BITS>(w, lane);
      const int channel = 32 * part + lane;
#pragma unroll
      for (int t = 0; t < 32; t += 16) {
        if (T == 32 && t) break;
        const int from = t ? from1 : from0, p = t ? page1 : page0;
        if (from >= T || base + t >= len || p < 0) continue;
        uint8_t* to = plane + (size_t)p * c.page_bytes + (size_t)head * c.head_bytes + sh.values +
                      ((size_t)(((base + t) & (c.page - 1)) / T) * io.head_dim + channel) * (T * BITS / 8);
        if (BITS == 8)
          store_chunk<4, 8>(to, w + (t ? BITS / 2 : 0), from);
        else if (T == 32)
          store_chunk<4, 4>(to, w, from);
        else
          store_chunk<2, 4>(to, w + (t ? BITS / 2 : 0), from);
      }
    }
  }
}

// ---------------------------------------------------------------------- read
template <int BITS, bool FP16>
__global__ void __launch_bounds__(kIoThreads, 4) read_kernel(const QuantIo io, const QuantShape sh,
                                                             const QuantJobs jb) {
  constexpr int W = BITS == 8 ? 8 : 4;  // words of a lane's 32 codes
  const CacheView& c = io.cache;
  const int lane = threadIdx.x & 31;
  const bool values = blockIdx.y;
  uint8_t* out = reinterpret_cast<uint8_t*>(const_cast<void*>(values ? io.V : io.K));
  const uint8_t* plane = c.pool + (BITS == 16 ? 2 * io.layer + values : io.layer) * c.plane_bytes;
  for (int job = blockIdx.x * kIoWarps + threadIdx.x / 32; job < jb.jobs; job += gridDim.x * kIoWarps) {
    const int unit = jb.per_job == 1 ? job / jb.parts : job;
    const int part0 = jb.per_job == 1 ? job - unit * jb.parts : 0, part_end = part0 + jb.per_job;
    const int bh = unit / jb.spans, span = unit - bh * jb.spans;
    const int b = bh / c.n_kv_heads, head = bh - b * c.n_kv_heads;
    const int s = io.slots[b];
    int first = io.first ? io.first[b] : 0, n = io.count ? io.count[b] : io.rows;
    int len = 0;
    if (s >= 0) {
      len = s < c.n_slots ? c.lens[s] : -1;
      if (len < 0 || len > c.max_len || first < 0 || first > c.max_len || n < 0 || n > io.rows) {
        if (lane == 0) fault(c, kStatusBadCache);
        len = 0;
      }
    }
    if (len == 0) first = n = 0;  // zeros only
    const int base = (first & ~31) + 32 * span;
    if (base - first >= io.rows) continue;
    const int pos = base + lane, i = pos - first;
    int page = -1;
    if (i >= 0 && i < n && pos < len) {
      page = c.table[(size_t)s * c.max_pages + (pos >> c.page_shift)];
      if (!valid_page(c, page)) {
        fault(c, kStatusBadCache);
        page = -1;
      }
    }
    const bool row_on = i >= 0 && i < io.rows;
    uint8_t* to = out + (((size_t)bh * io.rows + (row_on ? i : 0)) * io.head_dim + 32 * part0) * 2;
    const int off = pos & (c.page - 1);
    const uint8_t* block = plane + (size_t)max(page, 0) * c.page_bytes + (size_t)head * c.head_bytes;
    // Where this lane's codes of the first channels lie, and how far it is to the
    // next ones; for values (a lane is a channel) those of tokens 0 .. 15 and 16
    // .. 31, or of all, through the page of a token that is read.
    const int T = BITS == 8 || c.page == 16 ? 16 : 32;
    const uint8_t *at = block, *at2 = block;
    int step = 0;
    bool there = page >= 0, there2 = page >= 0;
    if (BITS == 16) {
      at += (size_t)off * c.row_bytes + 64 * part0;
      step = 64;
    } else if (!values) {
      at += ((size_t)part0 * (BITS / 4) * c.page + off) * 16;
      at2 = at + c.page * 16;
      step = BITS / 4 * c.page * 16;
    } else {
      const uint32_t sound = __ballot_sync(0xffffffffu, page >= 0);
      const uint32_t low = T == 32 ? sound : sound & 0xffffu, high = sound >> 16;
      there = low != 0;
      there2 = high != 0;
      const int p0 = __shfl_sync(0xffffffffu, page, low ? __ffs(low) - 1 : 0);
      const int p1 = __shfl_sync(0xffffffffu, page, high ? 15 + __ffs(high) : 0);
      const int piece = T * BITS / 8;
      const uint8_t* rest = plane + (size_t)head * c.head_bytes + sh.values + (32 * part0 + lane) * piece;
      at = rest + (size_t)max(p0, 0) * c.page_bytes + (size_t)((base & (c.page - 1)) / T) * io.head_dim * piece;
      at2 = rest + (size_t)max(p1, 0) * c.page_bytes + (size_t)(((base + 16) & (c.page - 1)) / T) * io.head_dim * piece;
      step = 32 * piece;
    }
    const int scale_step = values ? 2 * c.page : 2;
    const uint8_t* scales =
        block +
        (values ? sh.value_scales + 2 * part0 * c.page + off : sh.key_scales + off * sh.key_scale_bytes + 2 * part0);
    uint4 y[4] = {};
    uint32_t w[W] = {}, s0 = 0, s1 = 0;
    auto load = [&]() {  // of 32 channels
      if constexpr (BITS == 16) {
        if (there) {
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = __ldg(reinterpret_cast<const uint4*>(at) + k);
        }
      } else {
        if (BITS == 8) {
          if (there) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(at);
          if (there2) *reinterpret_cast<uint4*>(w + W - 4) = *reinterpret_cast<const uint4*>(at2);
        } else if (!values || T == 32) {
          if (there) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(at);
        } else {
          if (there) *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(at);
          if (there2) *reinterpret_cast<uint2*>(w + 2) = *reinterpret_cast<const uint2*>(at2);
        }
        if (page >= 0) {
          s0 = scales[0];
          s1 = scales[values ? c.page : 1];
        }
      }
      at += step;
      at2 += step;
      scales += scale_step;
    };
    load();
#pragma unroll 1
    for (int part = part0; part < part_end; ++part) {
      if constexpr (BITS == 16) {
        if (row_on) store_row(to, jb.wide, y);
        if (part + 1 < part_end) load();
      } else {
        uint32_t codes[W];
#pragma unroll
        for (int k = 0; k < W; ++k) codes[k] = w[k];
        const uint32_t scale0 = s0, scale1 = s1;
        if (part + 1 < part_end) load();  // the next channels are on their way meanwhile
        if (values) transpose_codes<BITS == 8 ? 8 : 4>(codes, lane);
        uint32_t v[8];
        decode_group<BITS, FP16>(codes, scale0, v);
        y[0] = make_uint4(v[0], v[1], v[2], v[3]);
        y[1] = make_uint4(v[4], v[5], v[6], v[7]);
        decode_group<BITS, FP16>(codes + W / 2, scale1, v);
        y[2] = make_uint4(v[0], v[1], v[2], v[3]);
        y[3] = make_uint4(v[4], v[5], v[6], v[7]);
        if (page < 0) y[0] = y[1] = y[2] = y[3] = make_uint4(0, 0, 0, 0);
        if (row_on) store_row(to, jb.wide, y);
      }
      to += 64;
    }
  }
}

QuantShape quant_shape(const QuantIo& io) {
  const int bits = io.cache.bits, page = io.cache.page;
  QuantShape sh;
  sh.key_scales = q_key_scales_at(bits, io.head_dim, page);
  sh.values = q_values_at(bits, io.head_dim, page);
  sh.value_scales = q_value_scales_at(bits, io.head_dim, page);
  sh.key_scale_bytes = q_key_scale_bytes(io.head_dim);
  return sh;
}

// All channels a job while that keeps every SM's warps busy, 32 of them else.
QuantJobs quant_jobs(const QuantIo& io) {
  QuantJobs jb;
  jb.parts = io.head_dim / 32;
  jb.spans = spans_of(io.rows);
  jb.jobs = io.batch * io.cache.n_kv_heads * jb.spans;
  jb.per_job = jb.parts;
  if (jb.jobs < 16 * io.sm_count) {
    jb.jobs *= jb.parts;
    jb.per_job = 1;
  }
  jb.wide = ((reinterpret_cast<uintptr_t>(io.K) | reinterpret_cast<uintptr_t>(io.V)) & 31) == 0;
  return jb;
}

// Blocks of keys, and as many of values: twice what stays resident (with no more
// than that 2 x 32K tokens stored and read back take 130 us as well, but 256 x 5
// drafted tokens 28.8 instead of 25.8).
int io_blocks(const QuantIo& io, const QuantJobs& jb) {
  return std::min((jb.jobs - 1) / kIoWarps + 1, 4 * io.sm_count);
}

}  // namespace

cudaError_t launch_kvq_write(const QuantIo& io, cudaStream_t stream) {
  auto kernel = io.cache.bits == 4 ? (io.fp16 ? quant_write_kernel<4, true> : quant_write_kernel<4, false>)
                                   : (io.fp16 ? quant_write_kernel<8, true> : quant_write_kernel<8, false>);
  const int smem = io.batch > 1 ? 2 * ((io.cache.n_slots + 31) / 32) * 4 : 0;
  if (smem > 40 * 1024) {
    cudaError_t e =
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlots / 32 * 2 * 4);
    if (e != cudaSuccess) return e;
  }
  const QuantJobs jb = quant_jobs(io);
  kernel<<<dim3(io_blocks(io, jb), 2), kIoThreads, smem, stream>>>(io, quant_shape(io), jb);
  return cudaGetLastError();
}

cudaError_t launch_kv_read(const QuantIo& io, cudaStream_t stream) {
  auto kernel = io.cache.bits == 4   ? (io.fp16 ? read_kernel<4, true> : read_kernel<4, false>)
                : io.cache.bits == 8 ? (io.fp16 ? read_kernel<8, true> : read_kernel<8, false>)
                                     : read_kernel<16, true>;
  const QuantJobs jb = quant_jobs(io);
  kernel<<<dim3(io_blocks(io, jb), 2), kIoThreads, 0, stream>>>(io, quant_shape(io), jb);
  return cudaGetLastError();
}

}  // namespace wise
