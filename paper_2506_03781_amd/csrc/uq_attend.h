// Device helpers of the attentions over the paged cache: matrix products of
// 16 x 16 tiles, the rows of a cache as their operands, sums over a wavefront.
// gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "uq_kv.h"
#include "uq_launch.h"

namespace uq {

namespace {

typedef __bf16 bf16x8d __attribute__((ext_vector_type(8)));
typedef float f32x4d __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4d __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2d __attribute__((ext_vector_type(2)));
typedef short s16x4d __attribute__((ext_vector_type(4)));

constexpr float LOG2E_D = 1.44269504088896341f;
constexpr float LOWEST = -3.402823466e38f;  // the running maximum before any position
constexpr float BF16_DOWN = 0x1p-24f;       // weights of a bf16 cache's values (codes have their own powers of two)
constexpr float BF16_BACK = 0x1p24f;
constexpr float MORE = 1.0f + 0x1p-17f;     // a weight's second term is MORE times it, less the first term
constexpr float SLACK = 8.0f;               // scores may exceed the reference by this (weights up to 2^8)
constexpr int WAVES = 4;
constexpr int STEP = 32;                    // positions of a wavefront's step
constexpr int CUS = 256;

__device__ __forceinline__ f32x4d mfma16(const u32x4d& a, const u32x4d& b, const f32x4d& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8d, a), __builtin_bit_cast(bf16x8d, b), c, 0,
                                                 0, 0);
}

__device__ __forceinline__ f32x4d mfma16(const u32x2d& a, const u32x2d& b, const f32x4d& c) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4d, a), __builtin_bit_cast(s16x4d, b), c, 0, 0,
                                                   0);
}

// Upper halves of two words: the bf16 values that a and b truncate to, a first.
__device__ __forceinline__ uint32_t top_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}

// Over the four lanes l % 16 + 16 k, in every one of them: a swap of rows (of
// halves) of x with itself leaves each row (half) beside its partner's copy.
template <typename Op>
__device__ __forceinline__ float over4(float x, Op op) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(op(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float max4(float x) {
  return over4(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum4(float x) {
  return over4(x, [](float a, float b) { return a + b; });
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Inclusive sums over the wavefront's lanes.
template <typename T>
__device__ __forceinline__ T wave_scan(T x) {
  static_assert(sizeof(T) == 4, "");
  auto add = [](T a, int moved) { return a + __builtin_bit_cast(T, moved); };
  x = add(x, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x111, 0xF, 0xF, false));  // row_shr:1
  x = add(x, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x112, 0xF, 0xF, false));
  x = add(x, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x114, 0xF, 0xF, false));
  x = add(x, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x118, 0xF, 0xF, false));
  x = add(x, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x142, 0xA, 0xF, false));  // row_bcast:15
  x = add(x, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x143, 0xC, 0xF, false));  // row_bcast:31
  return x;
}

// Element i of an array that no kernel running now writes, i the same in every
// lane: a scalar load, which does not wait for the vector loads before it.
__device__ __forceinline__ int scalar(const int32_t* p, int64_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p))[i];
}

template <int FMT, int D>
struct Form {
  static constexpr int ROW = FMT == KV_BF16 ? 2 * D : FMT == KV_U8 ? D : D / 2;  // bytes of a position
  static constexpr int KW = ROW / 16;               // words of a lane's quarter of a key row
  static constexpr int VB = ROW / 16;               // bytes of a lane's sixteenth of a value row
  static constexpr int VW = VB < 4 ? 1 : VB / 4;    // words
  static constexpr int NC = D / 32;                 // contraction steps of the scores
  static constexpr int NV = D / 16;                 // channel tiles of the output
};

template <int FMT, int D>
__device__ __forceinline__ void load_key(const char* __restrict__ tile, int lane, uint32_t (&w)[Form<FMT, D>::KW]) {
  using F = Form<FMT, D>;
  const char* row = tile + (lane & 15) * F::ROW;
  const int grp = lane >> 4;
  if constexpr (FMT == KV_BF16) {
#pragma unroll
    for (int c = 0; c < F::NC; ++c) {
      const u32x4d v = *reinterpret_cast<const u32x4d*>(row + 64 * c + 16 * grp);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * c + i] = v[i];
    }
  } else if constexpr (F::KW >= 4) {
#pragma unroll
    for (int c = 0; c < F::KW / 4; ++c) {
      const u32x4d v = *reinterpret_cast<const u32x4d*>(row + 4 * F::KW * grp + 16 * c);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * c + i] = v[i];
    }
  } else {
    const u32x2d v = *reinterpret_cast<const u32x2d*>(row + 4 * F::KW * grp);
    w[0] = v[0];
    w[1] = v[1];
  }
}

// The eight channels of contraction step c of a key as bf16.
template <int FMT, int D>
__device__ __forceinline__ u32x4d key_step(const uint32_t (&w)[Form<FMT, D>::KW], int c) {
  u32x4d a;
  if constexpr (FMT == KV_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = w[4 * c + i];
  } else if constexpr (FMT == KV_U8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(0u, w[2 * c + i / 2], i & 1 ? 0x0C030C02u : 0x0C010C00u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = w[c] >> (8 * (i / 2)) & (i & 1 ? 0x00F000F0u : 0x000F000Fu);
  }
  return a;
}

template <int FMT, int D>
__device__ __forceinline__ void load_value(const char* __restrict__ tile, int row, int lane,
                                           uint32_t (&w)[Form<FMT, D>::VW]) {
  using F = Form<FMT, D>;
  const char* at = tile + row * F::ROW + (lane & 15) * F::VB;
  if constexpr (F::VB == 16) {
    const u32x4d v = *reinterpret_cast<const u32x4d*>(at);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = v[i];
  } else if constexpr (F::VB == 8) {
    const u32x2d v = *reinterpret_cast<const u32x2d*>(at);
    w[0] = v[0];
    w[1] = v[1];
  } else if constexpr (F::VB == 4) {
    w[0] = *reinterpret_cast<const uint32_t*>(at);
  } else {
    w[0] = *reinterpret_cast<const uint16_t*>(at);
  }
}

// Two positions' values at the lane's channel c, as bf16.
template <int FMT, int D>
__device__ __forceinline__ uint32_t value_pair(const uint32_t (&a)[Form<FMT, D>::VW],
                                               const uint32_t (&b)[Form<FMT, D>::VW], int c) {
  if constexpr (FMT == KV_BF16) {
    return c & 1 ? top_halves(a[c / 2], b[c / 2]) : low_halves(a[c / 2], b[c / 2]);
  } else if constexpr (FMT == KV_U8) {
    return __builtin_amdgcn_perm(b[c / 4], a[c / 4], 0x0C040C00u + 0x00010001u * uint32_t(c & 3));
  } else {
    const uint32_t x = __builtin_amdgcn_perm(b[0], a[0], 0x0C040C00u + 0x00010001u * uint32_t(c / 2));
    return x & (c & 1 ? 0x00F000F0u : 0x000F000Fu);
  }
}

// bf16 pair (lo, hi) of two values, truncated.
__device__ __forceinline__ uint32_t pair(float lo, float hi) { return top_halves(__float_as_uint(lo), __float_as_uint(hi)); }

}  // namespace

}  // namespace uq
