// Device helpers of the paged key/value cache (layout in uniquan.h): where a
// position lies, and bf16 rounding towards either infinity.  gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "uq_launch.h"

namespace uq {

// Grid of n workgroups, n up to 2^35 (a dimension's work items count in 32
// bits), and the number of the running one, which may be n or more.
inline dim3 grid_of(int64_t n) {
  const int64_t x = n < (int64_t(1) << 20) ? n : int64_t(1) << 20;
  return dim3(unsigned(x), unsigned((n + x - 1) / x));
}
__device__ __forceinline__ int64_t workgroup() { return int64_t(blockIdx.y) * gridDim.x + blockIdx.x; }

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
