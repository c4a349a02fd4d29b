// Device helpers of the paged key/value cache (layout in uniquan.h): where a
// position lies, and bf16 rounding towards either infinity.  gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "uq_launch.h"

namespace uq {

// Page that holds position pos of sequence s, or -1: pos is in
// [0, max_pages page_len), and the table's entry may be anything.
__device__ __forceinline__ int kv_page(const KvCache& c, int64_t s, int pos) {
  const int p = c.pages[s * c.max_pages + (pos >> c.log_page)];
  return p >= 0 && p < c.n_pages ? p : -1;
}

// Largest bf16 value <= x, as fp32 (NaN stays NaN).
__device__ __forceinline__ float bf16_down(float x) {
  const uint32_t b = __float_as_uint(x) & 0xFFFF0000u;
  return __uint_as_float(b) > x ? __uint_as_float(b + 0x10000u) : __uint_as_float(b);
}

// Smallest bf16 value >= x for x >= 0, as fp32.
__device__ __forceinline__ float bf16_up(float x) {
  const uint32_t b = __float_as_uint(x) & 0xFFFF0000u;
  return __uint_as_float(b) < x ? __uint_as_float(b + 0x10000u) : __uint_as_float(b);
}

}  // namespace uq
