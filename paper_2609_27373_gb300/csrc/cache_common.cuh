// Device helpers of the calls that work on a paged cache.
#pragma once

#include "internal.cuh"

namespace wise {

__device__ __forceinline__ void fault(const CacheView& c, int bits) { atomicOr(c.status, bits); }

__device__ __forceinline__ bool valid_page(const CacheView& c, int page) { return page >= 0 && page < c.n_pages; }

__device__ __forceinline__ int pages_of(const CacheView& c, int len) { return (len + c.page - 1) / c.page; }

// Marks slots listed twice in bitmaps over the slots in shared memory; the second
// one, behind the first, is the result.  Ends with a barrier.
__device__ __forceinline__ const uint32_t* mark_twice(const CacheView& c, const int32_t* slots, int n, uint32_t* seen) {
  const int words = (c.n_slots + 31) / 32;
  uint32_t* twice = seen + words;
  for (int k = threadIdx.x; k < 2 * words; k += blockDim.x) seen[k] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int s = slots[i];
    if (s >= 0 && s < c.n_slots) {
      const uint32_t bit = 1u << (s & 31);
      if (atomicOr(&seen[s >> 5], bit) & bit) atomicOr(&twice[s >> 5], bit);
    }
  }
  __syncthreads();
  return twice;
}

}  // namespace wise
