// Attention of one new token per sequence over the paged key/value cache
// (uniquan_attn_decode); layout, formulas and errors in uniquan.h.
//
// Split.  A workgroup of four wavefronts takes one sequence, one key/value
// head, up to HEADS of its query heads and one chunk of the positions; its
// wavefronts take steps of 32 positions in turn, each with a running maximum
// and sum, and are joined in LDS.  The chunk length follows from all lengths
// (plan_slot): as many chunks as fill the GPU, of equal size within a
// sequence.  A sequence of one chunk is finished here, the others' chunks are
// joined by attn_join_kernel.
//
// One step, v_mfma_f32_16x16x32_bf16 (C[m][n] += A[m][k] B[k][n]; lane l
// supplies row l % 16 of A and column l % 16 of B at k = 8 (l / 16) .. + 8 and
// holds rows 4 (l / 16) .. + 4 of column l % 16 of C):
//   S^T = K Q^T    16 positions x 16 heads a tile, two tiles a step.  The
//                  keys' rows are read as they lie, 16 lanes a row.
//   O^T += V^T P^T 16 channels x 16 heads a tile, 32 positions deep.  Slot
//                  8 (l / 16) + j of the contraction is position
//                  4 (l / 16) + j % 4 of tile j / 4: those whose scores the
//                  lane holds, so P needs no exchange; and the lane reads
//                  those eight rows of V, 16 lanes a row, each its D / 16
//                  channels, and transposes them in registers.
// The heads are columns in both products, so maximum, sum and rescaling are
// per lane.  No data passes through LDS before the join.
//
// Precision.  Scores are fp32 sums of exact products.  A weight p (times the
// group's scale for codes) enters the second product as two bf16 terms, the
// truncated value and the truncated rest, so what is lost is below 2^-16 of
// it: with up to 8 heads the rest stands in the columns 8..15, which costs
// nothing, above that in a second product.  Codes are fed as c, 4-bit ones as
// 128 + c (one AND-OR makes two of them); the 128 leaves the scores through
// the product's start value -128 sum q.  In the output every step takes the
// codes' middle away again with the same bf16 terms (a product with a
// constant), and the exact weights carry the middle's value: what truncation
// takes off the terms then scales values around zero, not their offset, which
// in a long row is hundreds of times the output.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "uq_device.h"
#include "uq_kv.h"
#include "uq_launch.h"

namespace uq {

namespace {

typedef __bf16 bf16x8d __attribute__((ext_vector_type(8)));
typedef float f32x4d __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4d __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2d __attribute__((ext_vector_type(2)));

constexpr float LOG2E_D = 1.44269504088896341f;
constexpr float LOWEST = -3.402823466e38f;  // the running maximum before any position
constexpr float SLACK = 8.0f;               // scores may exceed the reference by this (weights up to 2^8)
constexpr int WAVES = 4;
constexpr int STEP = 32;                    // positions of a wavefront's step
constexpr int MIN_STEPS = 8;                // steps of the shortest chunk
constexpr int TARGET = 1024;                // workgroups that a split aims at
constexpr int MAX_SPLIT_SEQ = 4096;         // sequences up to which chunks are laid out

__device__ __forceinline__ f32x4d mfma16(const u32x4d& a, const u32x4d& b, const f32x4d& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8d, a), __builtin_bit_cast(bf16x8d, b), c, 0,
                                                 0, 0);
}

// Upper halves of two words: the bf16 values that a and b truncate to, a first.
__device__ __forceinline__ uint32_t top_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}

// Over the four lanes l % 16 + 16 k, in every one of them.
__device__ __forceinline__ float max4(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum4(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// ---------------------------------------------------------------------------
// which chunk a workgroup takes
// ---------------------------------------------------------------------------
struct Slot {
  int64_t s;      // sequence, or -1: none
  int chunk, n;   // its chunk and their number
  int64_t first;  // slot of the sequence's first chunk
  int len;
};

__device__ __forceinline__ int capped_len(const AttnDecodeLaunch& p, int64_t s) {
  const int64_t cap = p.c.max_pages << p.c.log_page;
  const int len = p.lens[s];
  return len < 0 ? 0 : int(len < cap ? len : cap);
}

__device__ __forceinline__ int64_t wave_sum64(int64_t x) {
  for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
  return x;
}
__device__ __forceinline__ int64_t wave_scan64(int64_t x, int lane) {
  for (int m = 1; m < 64; m <<= 1) {
    const int64_t y = __shfl_up(x, m);
    if (lane >= m) x += y;
  }
  return x;
}

// Slot `at` (or, by_seq, the slots of sequence `at`) of the chunks laid out in
// the sequences' order.  With all lengths in steps of 32 and their sum T, a
// chunk has at most c = max(MIN_STEPS, ceil(T / want)) steps, so there are at
// most want + n_seq of them; a sequence has ceil(steps / c), one at least.
// Every wavefront works it out by itself: the lanes take runs of the sequences.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(uint32_t(x))))) | uint64_t(uint32_t(uniform(int(x >> 32)))) << 32);
}
__device__ Slot plan_slot(const AttnDecodeLaunch& p, int64_t at, bool by_seq, int want) {
  const int lane = threadIdx.x & 63;
  const int64_t n = p.c.n_seq;
  Slot r{-1, 0, 1, at, 0};
  if (want == 0) {  // not split: slot and sequence are one
    if (at < n) {
      r.s = at;
      r.len = capped_len(p, at);
    }
    return r;
  }
  const int64_t per = (n + 63) / 64;
  int64_t total = 0;
  for (int64_t j = lane * per; j < lane * per + per && j < n; ++j) total += (capped_len(p, j) + STEP - 1) / STEP;
  total = wave_sum64(total);
  const int64_t c = std::max<int64_t>(MIN_STEPS, (total + want - 1) / want);
  auto chunks = [&](int64_t j) -> int64_t {
    if (j >= n) return 0;
    const int64_t k = ((capped_len(p, j) + STEP - 1) / STEP + c - 1) / c;
    return k > 1 ? k : 1;
  };
  int64_t mine = 0;
  for (int64_t j = lane * per; j < lane * per + per && j < n; ++j) mine += chunks(j);
  int64_t upto = wave_scan64(mine, lane);
  int64_t run, before;  // the run of sequences that holds it, and the slots before the run
  if (by_seq) {
    run = at / per;
  } else {
    const uint64_t past = __ballot(upto > at);
    if (past == 0) return r;
    run = __builtin_ctzll(past);
  }
  before = __shfl(upto - mine, int(run));
  const int64_t j = run * per + lane;
  mine = lane < per ? chunks(j) : 0;
  upto = wave_scan64(mine, lane) + before;
  int in;
  if (by_seq) {
    in = int(at - run * per);
  } else {
    const uint64_t past = __ballot(upto > at);
    in = __builtin_ctzll(past);
  }
  r.s = uniform(run * per + in);
  r.n = uniform(int(__shfl(mine, in)));
  r.first = uniform(int64_t(__shfl(upto - mine, in)));
  r.chunk = by_seq ? 0 : int(at - r.first);
  r.len = uniform(capped_len(p, r.s));
  return r;
}

// ---------------------------------------------------------------------------
// one chunk
// ---------------------------------------------------------------------------
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

// The eight channels of contraction step c of a key as bf16 (4-bit codes as 128 + c).
template <int FMT, int D>
__device__ __forceinline__ u32x4d key_step(const uint32_t (&w)[Form<FMT, D>::KW], int c) {
  u32x4d a;
  if constexpr (FMT == KV_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = w[4 * c + i];
  } else if constexpr (FMT == KV_U8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = w[2 * c + i / 2] >> (16 * (i & 1));
      a[i] = top_halves(__float_as_uint(float(x & 255u)), __float_as_uint(float(x >> 8 & 255u)));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = (w[c] >> (4 * i) & 0x000F000Fu) | 0x43004300u;
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

// Two positions' values at the lane's channel c, as bf16 (4-bit codes as 128 + c).
template <int FMT, int D>
__device__ __forceinline__ uint32_t value_pair(const uint32_t (&a)[Form<FMT, D>::VW],
                                               const uint32_t (&b)[Form<FMT, D>::VW], int c) {
  if constexpr (FMT == KV_BF16) {
    return c & 1 ? top_halves(a[c / 2], b[c / 2]) : low_halves(a[c / 2], b[c / 2]);
  } else if constexpr (FMT == KV_U8) {
    const int sh = 8 * (c & 3);
    return top_halves(__float_as_uint(float(a[c / 4] >> sh & 255u)), __float_as_uint(float(b[c / 4] >> sh & 255u)));
  } else {
    const uint32_t x = c < 4 ? low_halves(a[0], b[0]) : top_halves(a[0], b[0]);
    return (x >> (4 * (c & 3)) & 0x000F000Fu) | 0x43004300u;
  }
}

// WIDE: 16 query heads a workgroup, else 8 with the weights' rests in the upper columns.
template <int FMT, int D, int NG, bool WIDE>
__global__ __launch_bounds__(256) void attn_decode_kernel(AttnDecodeLaunch p, int want, int rtiles) {
  using F = Form<FMT, D>;
  constexpr int HEADS = WIDE ? 16 : 8;
  constexpr bool CODES = FMT != KV_BF16;
  constexpr int NGA = CODES ? NG : 1;
  constexpr float MID = FMT == KV_U8 ? 128.0f : 8.0f;
  const KvCache& c = p.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  // consecutive workgroups go to the 8 XCDs in turn: the row tiles that read one head's cache 8 apart
  const int64_t b = blockIdx.x;
  const int64_t unit = b / (8 * rtiles) * 8 + b % 8;
  const int rt = int(b / 8 % rtiles);
  const Slot sl = plan_slot(p, unit / c.H_kv, false, want);
  if (sl.s < 0) return;
  const int64_t s = sl.s;
  const int g = int(unit % c.H_kv);
  const int grp_heads = p.H / c.H_kv;
  const int h_in = rt * HEADS + (col & (HEADS - 1));  // head within its key/value head's group
  const bool rest = !WIDE && col >= 8;
  const uint32_t cut = rest ? 0xFFFF0000u : 0u;

  // queries, and (codes) their sums over each group of channels
  u32x4d q[F::NC];
  float qsum[NGA];
  {
    const uint16_t* row = p.Q + s * p.ld_q + (int64_t(g) * grp_heads + h_in) * D + 8 * grp;
    float part[F::NC];
#pragma unroll
    for (int k = 0; k < F::NC; ++k) {
      q[k] = h_in < grp_heads ? *reinterpret_cast<const u32x4d*>(row + 32 * k) : u32x4d{0, 0, 0, 0};
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) t += __uint_as_float(q[k][i] << 16) + __uint_as_float(q[k][i] & 0xFFFF0000u);
      part[k] = t;
    }
    if constexpr (CODES) {
#pragma unroll
      for (int i = 0; i < NGA; ++i) {
        float t = 0.0f;
#pragma unroll
        for (int k = i * F::NC / NGA; k < (i + 1) * F::NC / NGA; ++k) t += part[k];
        qsum[i] = sum4(t);
      }
    } else {
      qsum[0] = 0.0f;
    }
  }
  const float cl = p.scale * LOG2E_D;

  const int steps = (sl.len + STEP - 1) / STEP;
  const int u0 = int(int64_t(steps) * sl.chunk / sl.n), u1 = int(int64_t(steps) * (sl.chunk + 1) / sl.n);

  f32x4d acc[F::NV] = {};
  float off[NGA] = {};  // sums of weight times the value of the codes' middle
  float m = LOWEST, l = 0.0f;

  const int32_t* pages = c.pages + s * c.max_pages;
  const char* kc = static_cast<const char*>(c.k);
  const char* vc = static_cast<const char*>(c.v);
  const uint32_t* ks = reinterpret_cast<const uint32_t*>(c.k_stat);
  const uint32_t* vs = reinterpret_cast<const uint32_t*>(c.v_stat);

  for (int u = u0 + wave; u < u1; u += WAVES) {
    // the step's two tiles: place in the cache and positions that take part
    int64_t at[2];
    int64_t sat[2];
    int nv[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int base = u * STEP + 16 * t;
      int page = -1;
      if (base < sl.len) page = pages[base >> c.log_page];
      const bool is = page >= 0 && page < c.n_pages;
      nv[t] = is ? (sl.len - base < 16 ? sl.len - base : 16) : 0;
      const int64_t ph = int64_t(is ? page : 0) * c.H_kv + g;
      const int place = is ? base & (c.page_len - 1) : 0;
      at[t] = (ph * c.page_len + place) * F::ROW;
      sat[t] = ph * NGA * c.page_len + place + 4 * grp;
    }
    if (nv[0] + nv[1] == 0) continue;
    uint32_t kw[2][F::KW], vw[8][F::VW];
    u32x4d kst[2][NGA], vst[2][NGA];
#pragma unroll
    for (int t = 0; t < 2; ++t) load_key<FMT, D>(kc + at[t], lane, kw[t]);
    if constexpr (CODES) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < NGA; ++i) {
          kst[t][i] = *reinterpret_cast<const u32x4d*>(ks + sat[t] + i * c.page_len);
          vst[t][i] = *reinterpret_cast<const u32x4d*>(vs + sat[t] + i * c.page_len);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) load_value<FMT, D>(vc + at[j / 4], 4 * grp + j % 4, lane, vw[j]);

    // scores of positions 4 grp + i of tile t
    float x[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (CODES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[t][i] = 0.0f;
#pragma unroll
        for (int e = 0; e < NGA; ++e) {
          const float start = FMT == KV_U4 ? -128.0f * qsum[e] : 0.0f;
          f32x4d a = {start, start, start, start};
#pragma unroll
          for (int k = e * F::NC / NGA; k < (e + 1) * F::NC / NGA; ++k) a = mfma16(key_step<FMT, D>(kw[t], k), q[k], a);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[t][i] = __builtin_fmaf(__uint_as_float(kst[t][e][i] << 16), a[i],
                                     __builtin_fmaf(__uint_as_float(kst[t][e][i] & 0xFFFF0000u), qsum[e], x[t][i]));
        }
      } else {
        f32x4d a = {};
#pragma unroll
        for (int k = 0; k < F::NC; ++k) a = mfma16(key_step<FMT, D>(kw[t], k), q[k], a);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[t][i] = a[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[t][i] *= cl;
    }
    if (nv[0] + nv[1] < 32) {  // positions that take no part: no weight, and nothing of theirs in the products
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = 4 * grp + j % 4 < nv[j / 4];
        x[j / 4][j % 4] = in ? x[j / 4][j % 4] : -__builtin_inff();
        if constexpr (CODES) {
#pragma unroll
          for (int e = 0; e < NGA; ++e) vst[j / 4][e][j % 4] = in ? vst[j / 4][e][j % 4] : 0u;
        } else {
#pragma unroll
          for (int i = 0; i < F::VW; ++i) vw[j][i] = in ? vw[j][i] : 0u;
        }
      }
    }
    // running maximum: the reference moves only when a score exceeds it by SLACK
    float mx = x[0][0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mx = fmaxf(mx, x[j / 4][j % 4]);
    mx = max4(mx);
    if (__any(mx > m + SLACK)) {
      const float m1 = fmaxf(m, mx);
      const float f = __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= f;
#pragma unroll
      for (int k = 0; k < F::NV; ++k) acc[k] *= f;
      if constexpr (CODES) {
#pragma unroll
        for (int e = 0; e < NGA; ++e) off[e] *= f;
      }
    }
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = __builtin_amdgcn_exp2f(x[j / 4][j % 4] - m);
      l += w[j];
    }
#pragma unroll
    for (int e = 0; e < NGA; ++e) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (CODES) {
          const uint32_t st = vst[j / 4][e][j % 4];
          const float sc = __uint_as_float(st << 16);
          y[j] = w[j] * sc;
          off[e] = __builtin_fmaf(w[j], __builtin_fmaf(sc, MID, __uint_as_float(st & 0xFFFF0000u)), off[e]);
        } else {
          y[j] = w[j];
        }
      }
      u32x4d hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t a = __float_as_uint(y[2 * i]), d = __float_as_uint(y[2 * i + 1]);
        if constexpr (WIDE) {
          hi[i] = top_halves(a, d);
          lo[i] = top_halves(__float_as_uint(y[2 * i] - __uint_as_float(a & 0xFFFF0000u)),
                             __float_as_uint(y[2 * i + 1] - __uint_as_float(d & 0xFFFF0000u)));
        } else {
          hi[i] = top_halves(__float_as_uint(y[2 * i] - __uint_as_float(a & cut)),
                             __float_as_uint(y[2 * i + 1] - __uint_as_float(d & cut)));
        }
      }
#pragma unroll
      for (int k = e * F::NV / NGA; k < (e + 1) * F::NV / NGA; ++k) {
        u32x4d a;
        if constexpr (CODES) {
          constexpr uint32_t z = FMT == KV_U8 ? 0xC300C300u : 0xC308C308u;  // -128; -136
          const u32x4d mid = {z, z, z, z};
          acc[k] = mfma16(mid, hi, acc[k]);
          if constexpr (WIDE) acc[k] = mfma16(mid, lo, acc[k]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = value_pair<FMT, D>(vw[2 * i], vw[2 * i + 1], k);
        acc[k] = mfma16(a, hi, acc[k]);
        if constexpr (WIDE) acc[k] = mfma16(a, lo, acc[k]);
      }
    }
  }

  // join the wavefronts: row of column `col` in the order tile, row of the tile
  constexpr int LD = D + 4;
  __shared__ __attribute__((aligned(16))) float so[WAVES][16][LD];
  __shared__ float sm[WAVES][16], ss[WAVES][16];
  l = sum4(l);
#pragma unroll
  for (int e = 0; e < NGA; ++e) {
    if constexpr (CODES) {
      off[e] = rest ? 0.0f : sum4(off[e]);
    }
#pragma unroll
    for (int k = e * F::NV / NGA; k < (e + 1) * F::NV / NGA; ++k)
      *reinterpret_cast<f32x4d*>(&so[wave][col][16 * k + 4 * grp]) = CODES ? acc[k] + off[e] : acc[k];
  }
  if (grp == 0) {
    sm[wave][col] = m;
    ss[wave][col] = l;
  }
  __syncthreads();
  // two neighbouring channels of one head a thread
  for (int o = threadIdx.x; o < HEADS * D / 2; o += 256) {
    const int h = o / (D / 2), ch = o % (D / 2) * 2;
    const int hh = rt * HEADS + h;
    if (hh >= grp_heads) break;
    const int i0 = CODES ? ch : ch % F::NV * 16 + ch / F::NV;
    const int i1 = CODES ? ch + 1 : i0 + 16;
    float top = sm[0][h];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) top = fmaxf(top, sm[v][h]);
    float t = 0.0f, a0 = 0.0f, a1 = 0.0f;
#pragma unroll
    for (int v = 0; v < WAVES; ++v) {
      const float f = __builtin_amdgcn_exp2f(sm[v][h] - top);
      float b0 = so[v][h][i0], b1 = so[v][h][i1];
      if constexpr (!WIDE) {
        b0 += so[v][h + 8][i0];
        b1 += so[v][h + 8][i1];
      }
      t += f * ss[v][h];
      a0 += f * b0;
      a1 += f * b1;
    }
    const int64_t head = int64_t(g) * grp_heads + hh;
    if (sl.n == 1) {
      const float r = t == 0.0f ? 0.0f : 1.0f / t;
      *reinterpret_cast<uint32_t*>(p.O + s * p.ld_o + head * D + ch) = pack_bf16x2(a0 * r, a1 * r);
      if (ch == 0 && p.lse) p.lse[s * p.H + head] = t == 0.0f ? -__builtin_inff() : top + __builtin_amdgcn_logf(t);
    } else {
      float* part = p.ws + ((sl.first + sl.chunk) * p.H + head) * (D + 4);
      *reinterpret_cast<float2*>(part + 4 + ch) = make_float2(a0, a1);
      if (ch == 0) *reinterpret_cast<float2*>(part) = make_float2(top, t);
    }
  }
}

// Joins the chunks of a sequence's head: D / 4 lanes a chunk, 256 / (D / 4)
// chunks at a time.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnDecodeLaunch p, int want) {
  constexpr int LANES = D / 4, PAR = 256 / LANES;
  const int64_t s = blockIdx.x / p.H;
  const int h = blockIdx.x % p.H;
  const Slot sl = plan_slot(p, s, true, want);
  if (sl.n == 1) return;
  const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
  const float* base = p.ws + (sl.first * p.H + h) * (D + 4);
  const int64_t ld = int64_t(p.H) * (D + 4);
  float m = LOWEST, t = 0.0f;
  f32x4d a = {};
  for (int k = row; k < sl.n; k += PAR) {
    const float2 ml = *reinterpret_cast<const float2*>(base + k * ld);
    const f32x4d o = *reinterpret_cast<const f32x4d*>(base + k * ld + 4 + 4 * lane);
    const float m1 = fmaxf(m, ml.x);
    const float f0 = __builtin_amdgcn_exp2f(m - m1), f1 = __builtin_amdgcn_exp2f(ml.x - m1);
    m = m1;
    t = t * f0 + ml.y * f1;
    a = a * f0 + o * f1;
  }
  __shared__ f32x4d so[PAR][LANES];
  __shared__ float sm[PAR], st[PAR];
  so[row][lane] = a;
  if (lane == 0) {
    sm[row] = m;
    st[row] = t;
  }
  __syncthreads();
  if (row) return;
  float top = sm[0];
  for (int k = 1; k < PAR; ++k) top = fmaxf(top, sm[k]);
  t = 0.0f;
  a = f32x4d{};
  for (int k = 0; k < PAR; ++k) {
    const float f = __builtin_amdgcn_exp2f(sm[k] - top);
    t += f * st[k];
    a += f * so[k][lane];
  }
  const float r = t == 0.0f ? 0.0f : 1.0f / t;
  *reinterpret_cast<uint2*>(p.O + s * p.ld_o + int64_t(h) * D + 4 * lane) =
      make_uint2(pack_bf16x2(a[0] * r, a[1] * r), pack_bf16x2(a[2] * r, a[3] * r));
  if (lane == 0 && p.lse) p.lse[s * p.H + h] = t == 0.0f ? -__builtin_inff() : top + __builtin_amdgcn_logf(t);
}

// Query heads a workgroup takes, and workgroups a key/value head's heads take.
int row_heads(int H, int H_kv) { return H / H_kv > 8 ? 16 : 8; }
int row_tiles(int H, int H_kv) {
  const int r = row_heads(H, H_kv);
  return (H / H_kv + r - 1) / r;
}

// Chunks aimed at for each key/value head's row tile (0: sequences are not
// split), and how many there can be.
struct Split {
  int want;
  int64_t slots;
};
Split split_of(int64_t n_seq, int H, int H_kv, int64_t max_pages, int page_len) {
  const int64_t steps = (max_pages * page_len + STEP - 1) / STEP;
  if (n_seq > MAX_SPLIT_SEQ || steps <= MIN_STEPS) return {0, n_seq};
  const int64_t want = std::max<int64_t>(1, TARGET / (int64_t(H_kv) * row_tiles(H, H_kv)));
  return {int(want), std::min(want + n_seq, n_seq * ((steps + MIN_STEPS - 1) / MIN_STEPS))};
}

template <int FMT, int D, int NG>
void launch_form(const AttnDecodeLaunch& p, const Split& sp, int rt, hipStream_t st) {
  const int64_t units = (sp.slots * p.c.H_kv + 7) / 8 * 8;
  const dim3 grid{unsigned(units * rt)};
  if (p.H / p.c.H_kv > 8)
    attn_decode_kernel<FMT, D, NG, true><<<grid, 256, 0, st>>>(p, sp.want, rt);
  else
    attn_decode_kernel<FMT, D, NG, false><<<grid, 256, 0, st>>>(p, sp.want, rt);
}

template <int D>
hipError_t launch_d(const AttnDecodeLaunch& p, hipStream_t st) {
  const Split sp = split_of(p.c.n_seq, p.H, p.c.H_kv, p.c.max_pages, p.c.page_len);
  const int rt = row_tiles(p.H, p.c.H_kv);
  if (p.c.format == KV_BF16)
    launch_form<KV_BF16, D, 1>(p, sp, rt, st);
  else if (p.c.format == KV_U8)
    p.c.group == D ? launch_form<KV_U8, D, 1>(p, sp, rt, st) : launch_form<KV_U8, D, D / 32>(p, sp, rt, st);
  else
    p.c.group == D ? launch_form<KV_U4, D, 1>(p, sp, rt, st) : launch_form<KV_U4, D, D / 32>(p, sp, rt, st);
  if (hipError_t e = hipGetLastError()) return e;
  if (sp.want) {
    attn_join_kernel<D><<<dim3(unsigned(p.c.n_seq * p.H)), 256, 0, st>>>(p, sp.want);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

size_t attn_decode_ws(int64_t n_seq, int H, int H_kv, int d, int64_t max_pages, int page_len) {
  const Split sp = split_of(n_seq, H, H_kv, max_pages, page_len);
  return sp.want ? size_t(sp.slots) * size_t(H) * size_t(d + 4) : 0;
}

hipError_t launch_attn_decode(const AttnDecodeLaunch& p, hipStream_t st) {
  return p.c.d == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace uq
