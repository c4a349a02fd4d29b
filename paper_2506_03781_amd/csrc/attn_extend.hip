// Attention of several query rows per sequence over the paged key/value cache
// (uniquan_attn_extend): parts of prompts, trees of drafts, windows; formulas and
// errors in uniquan.h.
//
// Split.  The rows of a sequence and the query heads of a key/value head are the
// columns of one product, m (H / H_kv) of them in the order row, head.  A
// workgroup of four wavefronts takes some columns (a tile) and all positions that
// its rows see, or a share of them.  Where the tiles are fewer than the GPU holds
// workgroups, and where some are much longer than others, they are cut into shares
// of about equal length, and attn_extend_join_kernel joins those; workgroups find
// their place by adding up all sequences' tiles and steps of 32 positions, or, where
// nothing is cut, by a search among the sequences' first rows.
//
// Few columns (attn_extend_kernel: 16 or 32).  One step is that of the single-token
// attention (attn_decode.hip): S^T = K Q^T and O^T += V^T P^T with the heads as
// columns, K and V straight from the cache into registers, codes fed as they are;
// a workgroup's wavefronts take every fourth step.  Bound by the loads: 64 x 8 rows
// over 8192 positions of 8 heads in bf16 (2.2 GB) in 374 us, 5.8 TB/s.
// Many columns (attn_extend_wide_kernel: 128).  Tiles of keys and values in LDS, read
// by four wavefronts with 32 columns each.  A wavefront's products wait for its weights
// and the other way round, and 64 KB of tiles and 256 registers leave two wavefronts a
// SIMD to cover that: 2 x 2048 rows behind 6144 positions, 32 heads over 8, in 605 us,
// 795 TFLOP/s.  columns_of says which is taken where; with four sequences or more, those
// of few columns among many have the first kernel's tiles beside the second's.
//
// What is seen.  A step in which some column does not see all 32 positions (its
// own end, a window's edge, a tree's drafts, the end of the sequence or a missing
// page) is masked entry by entry: scores to -infinity, weights to 0, and nothing
// of a value or a scale that is not finite where the weight is 0 (its products
// are 0, not NaN).  All other steps, nearly all of a long history, have no masks.
//
// Precision.  With 16 columns as in attn_decode.hip.  With more a weight enters the
// second product as one bf16 value, rounded to nearest (2^-8 of it at most, either
// way), as in the block's causal attention: a second term would double that product,
// which bounds such calls.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "uq_attend.h"
#include "uq_device.h"
#include "uq_kv.h"
#include "uq_launch.h"
#include "uq_tile.h"

namespace uq {

namespace {

constexpr int MIN_STEPS = 8;  // of a share

// ---------------------------------------------------------------------------
// which tile and share a workgroup takes
// ---------------------------------------------------------------------------
struct Seq {
  int first, m;  // rows
  int len;
};
__device__ __forceinline__ Seq seq_of(const AttnExtendLaunch& p, int first, int end, int len) {
  const int64_t m = int64_t(end) - first;
  return Seq{first, first < 0 || m < 0 ? 0 : int(m < p.T ? m : p.T), len};
}
__device__ __forceinline__ int capped(const AttnExtendLaunch& p, int len) {
  const int64_t cap = p.c.max_pages << p.c.log_page;
  return len < 0 ? 0 : int(len < cap ? len : cap);
}

template <int COLS>
struct Work {
  const AttnExtendLaunch& p;
  int G;  // query heads of a key/value head
  __device__ __forceinline__ int tiles(const Seq& s) const {
    const int64_t cols = int64_t(s.m) * G;
    return cols < p.from_cols || cols > p.to_cols ? 0 : int((cols + COLS - 1) / COLS);
  }
  // steps that a tile's rows see, about
  __device__ __forceinline__ int steps(const Seq& s) const {
    const int all = (capped(p, s.len) + STEP - 1) / STEP;
    if (p.window <= 0) return all;
    const int64_t near = (int64_t(p.sinks) + p.window + s.m) / STEP + 3;
    return near < all ? int(near) : all;
  }
};

struct Unit {
  int s;          // sequence
  int at;         // of the sequence's units
  int slot;       // of the workspace, where the sequence is cut
  int64_t total;  // steps of all tiles
  double rate;    // shares a step
  int target;
  // Shares of a tile of so many steps: floor(steps target / total), so that all sequences' cuts are no more than
  // are wanted, of MIN_STEPS at least.
  __device__ __forceinline__ int parts(int steps) const {
    int64_t n = int64_t(double(steps) * rate + 1e-6);
    n -= n * total > int64_t(steps) * target;
    return int(std::max<int64_t>(1, std::min<int64_t>(n, steps / MIN_STEPS)));
  }
};

// Unit x where no tile is cut.  Sequence s has the numbers from floor(row_start[s] G / COLS) + s on, as many as tiles
// or one more (floor(a + b) - floor(a) + 1 is ceil(b) at least), so that a search finds it.  Adding up all sequences'
// tiles in every workgroup takes time with their square: 4096 of one row, 8 heads and 128 positions 2.4 ms (so 0.56),
// 16384 of one head 4.0 (0.28).  Where only sequences of up to to_cols columns are taken, each has as many numbers as
// such a one has tiles.
template <int COLS>
__device__ __forceinline__ bool find_whole(const AttnExtendLaunch& p, int G, int64_t x, Unit& u) {
  const int lane = threadIdx.x & 63, n = int(p.c.n_seq);
  int s = 0;
  int64_t at;
  if (p.to_cols < INT64_MAX) {
    const int64_t per = (p.to_cols + COLS - 1) / COLS;
    if (x >= per * n) return false;
    s = int(x / per);
    at = x % per;
  } else {
    auto first = [&](int j) { return std::min<int64_t>(std::max(p.row_start[j], 0), p.T) * G / COLS + j; };
    for (int size = n; size > 1;) {  // it is one of the `size` from s on
      const int step = (size + 63) / 64;
      const uint64_t past = __ballot(lane * step < size && first(s + lane * step) <= x);
      if (!past) return false;
      const int k = 63 - __builtin_clzll(past);
      s += k * step;
      size = std::min(step, size - k * step);
    }
    at = x - first(s);
  }
  u = Unit{uniform(s), int(at), 0, 0, 0.0, 0};
  const Seq seq = seq_of(p, p.row_start[u.s], p.row_start[u.s + 1], 0);
  return at >= 0 && at < Work<COLS>{p, G}.tiles(seq);
}

// Unit x: a share of a tile, or with TILES a tile that is cut; false: there are fewer.
// target: shares that are wanted (0: no tile is cut).
template <int COLS, bool TILES>
__device__ __forceinline__ bool find(const AttnExtendLaunch& p, int G, int64_t x, int target, Unit& u) {
  if (target == 0) return find_whole<COLS>(p, G, x, u);
  const Work<COLS> w{p, G};
  const int lane = threadIdx.x & 63;
  const int n = int(p.c.n_seq), run = (n + 63) / 64;
  auto seq = [&](int j) { return seq_of(p, p.row_start[j], p.row_start[j + 1], p.lens[j]); };
  int64_t total = 0;
  for (int j = lane * run; j < lane * run + run && j < n; ++j) {
    const Seq s = seq(j);
    total += int64_t(w.tiles(s)) * w.steps(s);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1)
    total += int64_t(uint64_t(uint32_t(__shfl_xor(int(total >> 32), d))) << 32 | uint32_t(__shfl_xor(int(total), d)));
  u.total = int64_t(uint64_t(uint32_t(uniform(int(total >> 32)))) << 32 | uint32_t(uniform(int(total))));
  u.rate = double(target) / double(u.total > 0 ? u.total : 1);
  u.target = target;
  auto count = [&](int j, int& un, int& sp) {
    un = sp = 0;
    if (j >= n) return;
    const Seq s = seq(j);
    const int tiles = w.tiles(s), parts = u.parts(w.steps(s));
    sp = parts > 1 ? tiles * parts : 0;
    un = !TILES ? tiles * parts : parts > 1 ? tiles : 0;
  };
  int un = 0, sp = 0;
  for (int j = lane * run; j < lane * run + run; ++j) {
    int a, b;
    count(j, a, b);
    un += a;
    sp += b;
  }
  int upto = wave_scan(un), supto = wave_scan(sp);
  if (x >= __builtin_amdgcn_readlane(upto, 63)) return false;
  int in = __builtin_ctzll(__ballot(upto > int(x)));
  u.s = in * run;
  int before = __builtin_amdgcn_readlane(upto - un, in);
  u.slot = __builtin_amdgcn_readlane(supto - sp, in);
  if (run > 1) {
    for (const int end = u.s + run; u.s < end; u.s += 64) {
      const int j = u.s + lane < end ? u.s + lane : n;
      count(j, un, sp);
      upto = wave_scan(un) + before;
      supto = wave_scan(sp) + u.slot;
      const uint64_t past = __ballot(upto > int(x));
      if (past) {
        in = __builtin_ctzll(past);
        u.s += in;
        before = __builtin_amdgcn_readlane(upto - un, in);
        u.slot = __builtin_amdgcn_readlane(supto - sp, in);
        break;
      }
      before = __builtin_amdgcn_readlane(upto, 63);
      u.slot = __builtin_amdgcn_readlane(supto, 63);
    }
  }
  u.at = int(x) - before;
  return true;
}

// A share's sums for one column: (maximum, sum, -, -, D values) against that maximum.
template <int COLS, int D>
__device__ __forceinline__ float* part_of(const AttnExtendLaunch& p, int64_t slot, int g, int col) {
  return p.ws + ((slot * p.c.H_kv + g) * COLS + col) * (D + 4);
}

// Bits [at, at + 32) of a row's mask; at > -32, bits outside it 0.
__device__ __forceinline__ uint32_t mask_bits(const uint64_t* row, int words, int at) {
  const int w = at >> 6, sh = at & 63;
  const uint64_t lo = w >= 0 && w < words ? row[w] : 0u, hi = w + 1 >= 0 && w + 1 < words ? row[w + 1] : 0u;
  return uint32_t(sh ? lo >> sh | hi << (64 - sh) : lo);
}

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = std::min(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = std::max(x, __shfl_xor(x, d));
  return x;
}

// Whether one of a word's two bf16 values is not finite.
__device__ __forceinline__ bool wild(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// (Two workgroups a CU are the most for which nothing is spilled in the loop.)
template <int FMT, int D, int NG, int NT>
__global__ __launch_bounds__(256, 2) void attn_extend_kernel(AttnExtendLaunch p, int target) {
  using F = Form<FMT, D>;
  constexpr int COLS = 16 * NT;
  constexpr bool CODES = FMT != KV_BF16, TWO = NT == 1;  // two terms a weight
  constexpr float MID = FMT == KV_U8 ? 128.0f : 8.0f;
  constexpr float VSCALE = 0x1p64f;  // on the scales
  constexpr float VBACK = 0x1p69f;   // 2^133 / VSCALE
  auto sixteenfold = [](int k) { return FMT == KV_U4 && k % 2 == 1; };  // 4-bit codes of the odd channel tiles
  constexpr int LD = D + 4;
  __shared__ __attribute__((aligned(16))) float so[WAVES][16][LD];
  __shared__ float sm[WAVES][16], ss[WAVES][16];
  const KvCache& c = p.c;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int G = p.H / c.H_kv;
  const int64_t b = workgroup();
  const int g = int(b % c.H_kv);  // one key/value head's workgroups on one XCD, or on as few as can be
  Unit unit;
  if (!find<COLS, false>(p, G, b / c.H_kv, target, unit)) return;
  const int s = unit.s;
  const Seq seq = seq_of(p, scalar(p.row_start, s), scalar(p.row_start, s + 1), scalar(p.lens, s));
  const Work<COLS> work{p, G};
  const int tiles = work.tiles(seq), parts = unit.parts(work.steps(seq));
  const int part = unit.at / tiles, tile = tiles - 1 - unit.at % tiles;  // the longest first
  const int len = capped(p, seq.len);
  const int base = seq.len < 0 ? -seq.m : std::max(seq.len - seq.m, -seq.m);
  const bool tree = p.mask != nullptr;

  // the lane's columns: rows of Q and what they see
  int64_t row[NT];      // -1: none
  int head[NT];
  int end[NT], low[NT];  // seen: below end, at low or behind (or below sinks)
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t i = int64_t(tile) * COLS + 16 * n + col;
    const int j = int(i / G);
    row[n] = j < seq.m && int64_t(seq.first) + j < p.T ? int64_t(seq.first) + j : -1;
    head[n] = g * G + int(i % G);
    end[n] = tree ? base : base + j + 1;
    const int64_t at = row[n] >= 0 && p.pos ? p.pos[row[n]] : int64_t(base) + j;
    low[n] = p.window > 0 ? int(std::min<int64_t>(std::max<int64_t>(at - p.window + 1, 0), 0x7FFFFFFF)) : 0;
  }
  int end_min = 0x7FFFFFFF, end_max = 0, low_min = 0x7FFFFFFF, low_max = 0;
#pragma unroll
  for (int n = 0; n < NT; ++n)
    if (row[n] >= 0) {
      end_min = std::min(end_min, end[n]);
      end_max = std::max(end_max, end[n]);
      low_min = std::min(low_min, low[n]);
      low_max = std::max(low_max, low[n]);
    }
  end_min = uniform(wave_min(end_min));
  end_max = uniform(wave_max(end_max));
  low_min = uniform(wave_min(low_min));
  low_max = uniform(wave_max(low_max));

  // the steps of the tile: those with sinks, then from the window's begin to the last end
  const int hi = tree ? len : std::min(len, end_max);
  const int lo = std::max(0, tree ? std::min(low_min, base) : low_min);
  const int n_sink = p.window > 0 ? (std::min(p.sinks, std::max(hi, 0)) + STEP - 1) / STEP : 0;
  const int u_lo = std::max(lo / STEP, n_sink);
  const int n_steps = n_sink + std::max(0, (std::max(hi, 0) + STEP - 1) / STEP - u_lo);
  const int i0 = int(int64_t(n_steps) * part / parts), i1 = int(int64_t(n_steps) * (part + 1) / parts);
  auto step_at = [&](int i) { return i < n_sink ? i : u_lo + (i - n_sink); };

  const uint32_t page_bytes = uint32_t(c.H_kv) * uint32_t(c.page_len) * F::ROW;
  const uint32_t page_stats = uint32_t(c.H_kv) * uint32_t(c.page_len) * NG;
  const uint32_t head_bytes = uint32_t(g) * uint32_t(c.page_len) * F::ROW;
  const uint32_t lane_stat = (uint32_t(g) * NG + uint32_t(grp % NG)) * uint32_t(c.page_len) + col;
  uint32_t pick[NG], mids[NG];
#pragma unroll
  for (int e = 0; e < NG; ++e) {
    pick[e] = grp == e ? pair(VSCALE, 0.0f) : 0u;
    mids[e] = grp == e ? pair(MID, 1.0f) : 0u;
  }

  // The loads run a step ahead of the products, as in the single-token attention.
  struct Ahead {
    int i, u, page[2];
    uint64_t place[2], stat[2];
    int nv[2];  // positions of each tile that exist
  } next;
  uint32_t kw[2][F::KW], vw[8][F::VW], kst[2], vst[2];
  const int32_t* pages = c.pages + int64_t(s) * c.max_pages;
  auto look_up = [&] {
    next.u = step_at(next.i);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int at = next.u * STEP + 16 * t;
      next.page[t] = next.i < i1 && at < len ? scalar(pages, at >> c.log_page) : -1;
    }
  };
  auto load_keys = [&] {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int at = next.u * STEP + 16 * t;
      const bool is = next.page[t] >= 0 && next.page[t] < c.n_pages;
      const uint32_t pg = is ? uint32_t(next.page[t]) : 0u;
      const uint32_t r = is ? uint32_t(at & (c.page_len - 1)) : 0u;
      next.nv[t] = is ? std::min(16, len - at) : 0;
      next.place[t] = uint64_t(pg) * page_bytes + (head_bytes + r * F::ROW);
      next.stat[t] = uint64_t(pg) * page_stats + r;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      load_key<FMT, D>(static_cast<const char*>(c.k) + next.place[t], lane, kw[t]);
      if constexpr (CODES) kst[t] = (reinterpret_cast<const uint32_t*>(c.k_stat) + next.stat[t])[lane_stat];
    }
  };
  auto load_values = [&] {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if constexpr (CODES) vst[t] = (reinterpret_cast<const uint32_t*>(c.v_stat) + next.stat[t])[lane_stat];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      load_value<FMT, D>(static_cast<const char*>(c.v) + next.place[j / 4], 4 * grp + j % 4, lane, vw[j]);
    next.i += WAVES;
    look_up();
  };

  // queries, a negative scale's sign on them; for codes scaled, and their sums over each group of channels
  u32x4d q[NT][F::NC];
  u32x4d qs[NT] = {};
  float cl[NT];  // scores to exponents of 2
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const uint16_t* at = p.Q + (row[n] < 0 ? 0 : row[n]) * p.ld_q + int64_t(head[n]) * D + 8 * grp;
#pragma unroll
    for (int k = 0; k < F::NC; ++k)
      q[n][k] = row[n] >= 0 ? *reinterpret_cast<const u32x4d*>(at + 32 * k) : u32x4d{0, 0, 0, 0};
  }
  next.i = i0 + wave;
  look_up();
  load_keys();
  int nv[2] = {next.nv[0], next.nv[1]};
  load_values();
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    cl[n] = fabsf(p.scale) * LOG2E_D;
    if (p.scale < 0.0f) {
#pragma unroll
      for (int k = 0; k < F::NC; ++k) q[n][k] ^= 0x80008000u;
    }
    if constexpr (CODES) {
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < F::NC; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = std::max(top, std::max(q[n][k][i] << 16 & 0x7FFF0000u, q[n][k][i] & 0x7FFF0000u));
      const int ex = int(__float_as_uint(max4(__uint_as_float(top))) >> 23) - 127;
      const float up = ldexpf(1.0f, 120 - std::max(ex, -7));
      cl[n] = cl[n] * ldexpf(1.0f, 13 - 64 + std::max(ex, -7));  // 2^133 over the queries' power and the scales'
#pragma unroll
      for (int k = 0; k < F::NC; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          q[n][k][i] = pair(__uint_as_float(q[n][k][i] << 16) * up, __uint_as_float(q[n][k][i] & 0xFFFF0000u) * up);
      float mine = 0.0f;
#pragma unroll
      for (int e = 0; e < NG; ++e) {
        float t = 0.0f;
#pragma unroll
        for (int k = e * F::NC / NG; k < (e + 1) * F::NC / NG; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            t += __uint_as_float(q[n][k][i] << 16) * 0x1p-69f + __uint_as_float(q[n][k][i] & 0xFFFF0000u) * 0x1p-69f;
        t = sum4(t);
        if (grp == e) mine = t;
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const float h = __uint_as_float(__float_as_uint(mine) & 0xFFFF0000u);
        qs[n][i] = pair(0.0f, h);
        mine -= h;
      }
      if constexpr (FMT == KV_U4) {
#pragma unroll
        for (int k = 0; k < F::NC; ++k)
#pragma unroll
          for (int i = 1; i < 4; i += 2)
            q[n][k][i] = pair(__uint_as_float(q[n][k][i] << 16) * 0x1p-4f, __uint_as_float(q[n][k][i] & 0xFFFF0000u) * 0x1p-4f);
      }
    }
  }

  f32x4d acc[NT][F::NV] = {};
  f32x4d mid[NT][NG] = {};  // sums of the products' weights times minus the codes' middle
  float off[NT][NG] = {};   // sums of weight times the value of the codes' middle
  float m[NT], l[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n] = LOWEST;
    l[n] = 0.0f;
  }

  for (int i = i0 + wave; i < i1; i += WAVES) {
    const int t0 = step_at(i) * STEP;
    // scores of positions 4 grp + i of tile t
    float x[NT][8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4d sum[NT] = {};
      if constexpr (CODES) {
        const u32x4d st4 = {kst[t], kst[t], kst[t], kst[t]};
        const u32x2d st = {kst[t], kst[t]};
#pragma unroll
        for (int n = 0; n < NT; ++n) sum[n] = mfma16(st4, qs[n], sum[n]);  // the three terms at once
#pragma unroll
        for (int e = 0; e < NG; ++e) {
          f32x4d a[NT] = {};
#pragma unroll
          for (int k = e * F::NC / NG; k < (e + 1) * F::NC / NG; ++k) {
            const u32x4d ks = key_step<FMT, D>(kw[t], k);
#pragma unroll
            for (int n = 0; n < NT; ++n) a[n] = mfma16(ks, q[n][k], a[n]);
          }
          const f32x4d sc = mfma16(st, u32x2d{pick[e], 0u}, f32x4d{});
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[n][r] = __builtin_fmaf(sc[r], a[n][r], sum[n][r]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < F::NC; ++k) {
          const u32x4d ks = key_step<FMT, D>(kw[t], k);
#pragma unroll
          for (int n = 0; n < NT; ++n) sum[n] = mfma16(ks, q[n][k], sum[n]);
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[n][4 * t + r] = sum[n][r];
    }
    load_keys();
    const bool cut = nv[0] + nv[1] < STEP || t0 + STEP > end_min || (t0 < low_max && t0 + STEP > p.sinks);
    uint32_t seen[NT];  // bit j: position 4 grp + j % 4 of tile j / 4
    if (cut) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        uint32_t drafts = 0;
        if (tree && t0 + STEP > base && row[n] >= 0)
          drafts = mask_bits(p.mask + row[n] * p.words, p.words, t0 - base);
        seen[n] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int in = 16 * (j / 4) + 4 * grp + j % 4, at = t0 + in;
          const bool ok = at < end[n] ? (at >= low[n] || (p.window > 0 && at < p.sinks)) : (at >= base && (drafts >> in & 1));
          seen[n] |= ok && in - 16 * (j / 4) < nv[j / 4] ? 1u << j : 0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[n][j] = seen[n] >> j & 1 ? x[n][j] : -__builtin_inff();
      }
      // nothing of what does not exist
      if constexpr (!CODES) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int w = 0; w < F::VW; ++w) vw[j][w] = 4 * grp + j % 4 < nv[j / 4] ? vw[j][w] : 0u;
      }
    }
    float w[NT][8];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      // running maximum: the reference moves only when a score exceeds it by SLACK
      float mx = x[n][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, x[n][j]);
      mx = max4(mx) * cl[n];
      if (__any(mx > m[n] + SLACK)) {
        const float m1 = mx > m[n] + SLACK ? mx : m[n];  // a column's alone: rows do not depend on others
        const float f = __builtin_amdgcn_exp2f(m[n] - m1);
        m[n] = m1;
        l[n] *= f;
#pragma unroll
        for (int k = 0; k < F::NV; ++k) acc[n][k] *= f;
        if constexpr (CODES) {
#pragma unroll
          for (int e = 0; e < NG; ++e) {
            mid[n][e] *= f;
            off[n][e] *= f;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) w[n][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][j], cl[n], -m[n]));
      if (cut) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[n][j] = seen[n] >> j & 1 ? w[n][j] : 0.0f;
      }
      l[n] += ((w[n][0] + w[n][1]) + (w[n][2] + w[n][3])) + ((w[n][4] + w[n][5]) + (w[n][6] + w[n][7]));
    }
    // the weights as operands: two bf16 terms, or one rounded to nearest
    auto operands = [&](const float (&z)[8], u32x4d& h, u32x4d& lo) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (TWO) {
          auto less = [](float v) { return __builtin_fmaf(v, MORE, -__uint_as_float(__float_as_uint(v) & 0xFFFF0000u)); };
          h[r] = pair(z[2 * r], z[2 * r + 1]);
          lo[r] = pair(less(z[2 * r]), less(z[2 * r + 1]));
        } else {
          h[r] = pack_bf16x2(z[2 * r], z[2 * r + 1]);
        }
      }
    };
#pragma unroll
    for (int e = 0; e < NG; ++e) {
      u32x4d h[NT], lo2[NT];
      if constexpr (CODES) {
        f32x4d sc[2], md[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x2d st = {vst[t], 0u};
          sc[t] = mfma16(st, u32x2d{pick[e], 0u}, f32x4d{});
          md[t] = mfma16(st, u32x2d{mids[e], 0u}, f32x4d{});
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float z[8];
          if (cut) {  // scales that are not finite where the weight is 0
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              z[j] = w[n][j] == 0.0f ? 0.0f : w[n][j] * sc[j / 4][j % 4];
              off[n][e] += w[n][j] == 0.0f ? 0.0f : w[n][j] * md[j / 4][j % 4];
            }
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              z[j] = w[n][j] * sc[j / 4][j % 4];
              off[n][e] = __builtin_fmaf(w[n][j], md[j / 4][j % 4], off[n][e]);
            }
          }
          operands(z, h[n], lo2[n]);
          const uint32_t bits = FMT == KV_U8 ? 0x80808080u : 0x80088008u;  // minus the middle, as the codes
          const u32x4d minus = {bits, bits, bits, bits};
          mid[n][e] = mfma16(minus, h[n], mid[n][e]);
          if constexpr (TWO) mid[n][e] = mfma16(minus, lo2[n], mid[n][e]);
        }
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float z[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) z[j] = w[n][j] * BF16_DOWN;
          operands(z, h[n], lo2[n]);
        }
        if (cut) {
          // values that are not finite: out of the products, and in by themselves where there is a weight
          bool any = false;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int v = 0; v < F::VW; ++v) any |= wild(vw[j][v]);
          if (__any(any)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
#pragma unroll 1
              for (int src = 0; src < 4; ++src) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  const float z = __shfl(w[n][j], col + 16 * src) * BF16_DOWN;
#pragma unroll
                  for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int v = 0; v < F::VW; ++v) {
                      const uint32_t pairs = __shfl(vw[j][v], 4 * grp + r + 16 * src);
                      const float a = __uint_as_float(pairs << 16), b2 = __uint_as_float(pairs & 0xFFFF0000u);
                      if (z != 0.0f && a - a != 0.0f) acc[n][2 * v][r] += z * a;
                      if (z != 0.0f && b2 - b2 != 0.0f) acc[n][2 * v + 1][r] += z * b2;
                    }
                }
              }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int v = 0; v < F::VW; ++v) {
                if ((vw[j][v] & 0x7F80u) == 0x7F80u) vw[j][v] &= 0xFFFF0000u;
                if ((vw[j][v] & 0x7F800000u) == 0x7F800000u) vw[j][v] &= 0xFFFFu;
              }
          }
        }
      }
#pragma unroll
      for (int k = e * F::NV / NG; k < (e + 1) * F::NV / NG; ++k) {
        u32x4d a;
#pragma unroll
        for (int r = 0; r < 4; ++r) a[r] = value_pair<FMT, D>(vw[2 * r], vw[2 * r + 1], k);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc[n][k] = mfma16(a, h[n], acc[n][k]);
          if constexpr (TWO) acc[n][k] = mfma16(a, lo2[n], acc[n][k]);
        }
      }
    }
    nv[0] = next.nv[0];
    nv[1] = next.nv[1];
    load_values();
  }

  // join the wavefronts, a column tile at a time
  const bool whole = parts == 1;
  const int64_t slot = int64_t(unit.slot) + unit.at;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const float ln = sum4(l[n]);
    if (n) __syncthreads();
#pragma unroll
    for (int e = 0; e < NG; ++e) {
      const float o = CODES ? sum4(off[n][e]) : 0.0f;
#pragma unroll
      for (int k = e * F::NV / NG; k < (e + 1) * F::NV / NG; ++k) {
        f32x4d v = acc[n][k];
        if constexpr (CODES) v = sixteenfold(k) ? (v + mid[n][e] * 16.0f) * (VBACK / 16) + o : (v + mid[n][e]) * VBACK + o;
        *reinterpret_cast<f32x4d*>(&so[wave][col][16 * k + 4 * grp]) = v;
      }
    }
    if (grp == 0) {
      sm[wave][col] = m[n];
      ss[wave][col] = ln;
    }
    __syncthreads();
    // two neighbouring channels of a column a thread
    for (int o = threadIdx.x; o < 16 * D / 2; o += 256) {
      const int h = o / (D / 2), cn = o % (D / 2) * 2;
      const int64_t idx = int64_t(tile) * COLS + 16 * n + h;
      const int j = int(idx / G);
      const int64_t r = int64_t(seq.first) + j;
      if (j >= seq.m || r >= p.T) break;
      const int a0 = CODES ? cn : cn % F::NV * 16 + cn / F::NV;
      const int a1 = CODES ? cn + 1 : a0 + 16;
      float top = sm[0][h];
#pragma unroll
      for (int v = 1; v < WAVES; ++v) top = fmaxf(top, sm[v][h]);
      float t = 0.0f, x0 = 0.0f, x1 = 0.0f;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        const float f = __builtin_amdgcn_exp2f(sm[v][h] - top);
        t += f * ss[v][h];
        x0 += f * so[v][h][a0];
        x1 += f * so[v][h][a1];
      }
      if (whole) {
        const int hd = g * G + int(idx % G);
        const float inv = (CODES ? 1.0f : BF16_BACK) / t;
        // no weight at all: 0, where the values may have made the sums NaN
        *reinterpret_cast<uint32_t*>(p.O + r * p.ld_o + int64_t(hd) * D + cn) = t == 0.0f ? 0u : pack_bf16x2(x0 * inv, x1 * inv);
        if (cn == 0 && p.lse) p.lse[r * p.H + hd] = t == 0.0f ? -__builtin_inff() : top + __builtin_amdgcn_logf(t);
      } else if (slot < int64_t(target)) {
        float* out = part_of<COLS, D>(p, slot, g, 16 * n + h);
        *reinterpret_cast<float2*>(out + 4 + cn) = make_float2(x0, x1);
        if (cn == 0) *reinterpret_cast<float2*>(out) = make_float2(top, t);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// many columns: tiles in LDS, read by four wavefronts of 32 columns each
// ---------------------------------------------------------------------------
constexpr int WIDE = 128;  // columns of a workgroup

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }
__device__ __forceinline__ float max2(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// The codes of a thread's piece of a tile and their statistics, between their loads
// and LDS: row threadIdx.x / 8 of 32, codes 16 q .. + 16 as they lie (q = threadIdx.x % 8).
template <int FMT>
struct Codes {
  static constexpr int NG = 4;                    // groups of a head
  static constexpr int W = FMT == KV_U8 ? 4 : 2;  // words of 16 codes
  uint32_t k[W], v[W], ks[2], vs[NG];
  bool is;

  __device__ __forceinline__ void load(const KvCache& c, const uint64_t (&at)[2], const uint64_t (&st)[2],
                                       const int (&nv)[2]) {
    const int r = threadIdx.x >> 3, q = threadIdx.x & 7, t = r >> 4;
    is = (r & 15) < nv[t];
    const uint64_t o = at[t] + uint32_t(r & 15) * (FMT == KV_U8 ? 128u : 64u) + uint32_t(q) * (4 * W);
    if constexpr (FMT == KV_U8) {
      const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const char*>(c.k) + o);
      const uint4 b = *reinterpret_cast<const uint4*>(static_cast<const char*>(c.v) + o);
      k[0] = a.x; k[1] = a.y; k[2] = a.z; k[3] = a.w;
      v[0] = b.x; v[1] = b.y; v[2] = b.z; v[3] = b.w;
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const char*>(c.k) + o);
      const uint2 b = *reinterpret_cast<const uint2*>(static_cast<const char*>(c.v) + o);
      k[0] = a.x; k[1] = a.y;
      v[0] = b.x; v[1] = b.y;
    }
    const uint32_t* kst = reinterpret_cast<const uint32_t*>(c.k_stat) + st[t] + (r & 15);
    const uint32_t* vst = reinterpret_cast<const uint32_t*>(c.v_stat) + st[t] + (r & 15);
    const uint32_t len = uint32_t(c.page_len);
    // the piece's two runs of eight channels lie in groups 2 (q % 2) and the next
    ks[0] = kst[(2 * (q & 1)) * len];
    ks[1] = kst[(2 * (q & 1) + 1) * len];
#pragma unroll
    for (int e = 0; e < NG; ++e) vs[e] = vst[uint32_t(e) * len];
  }

  static __device__ __forceinline__ float code(const uint32_t (&w)[W], int i) {
    return float(FMT == KV_U8 ? w[i / 4] >> (8 * (i & 3)) & 255u : w[i / 8] >> (4 * (i & 7)) & 15u);
  }
  // Two values as two bf16 terms each.
  static __device__ __forceinline__ void terms(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf16x2(a, b);
    lo = pack_bf16x2(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xFFFF0000u));
  }
  static __device__ __forceinline__ float value(uint32_t st, float c) {
    return __builtin_fmaf(__uint_as_float(st << 16), c, __uint_as_float(st & 0xFFFF0000u));
  }

  // Into LDS: tiles kh, kl, vh, vl of the values' two terms; rows that do not exist are 0.
  __device__ __forceinline__ void store(u32x4a* stage) const {
    const int r = threadIdx.x >> 3, q = threadIdx.x & 7, rho = perm32(r);
    u32x4a* row = stage + rho * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // channels 32 cc + 8 (q / 2) .. + 8, cc = 2 (q % 2) + h
      u32x4a hi, lo;
      const uint32_t st = is ? ks[h] : 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (4-bit codes of a run lie in the order 0 2 4 6 1 3 5 7)
        const int a = 8 * h + (FMT == KV_U8 ? 2 * j : j), b = 8 * h + (FMT == KV_U8 ? 2 * j + 1 : j + 4);
        uint32_t x, y;
        terms(value(st, code(k, a)), value(st, code(k, b)), x, y);
        hi[j] = x;
        lo[j] = y;
      }
      const int chunk = (4 * (2 * (q & 1) + h) + (q >> 1)) ^ swz(rho);
      row[chunk] = hi;
      row[TILE16 + chunk] = lo;
    }
    uint32_t* vrow = reinterpret_cast<uint32_t*>(row + 2 * TILE16);
#pragma unroll
    for (int b = 0; b < 8; ++b) {  // channels 16 b + 2 q and the next
      uint32_t hi, lo;
      const uint32_t st = is ? vs[b / 2] : 0u;
      terms(value(st, code(v, b)), value(st, code(v, b + 8)), hi, lo);
      const int at = ((2 * b + (q >> 2)) ^ swz(rho)) * 4 + (q & 3);
      vrow[at] = hi;
      vrow[TILE16 * 4 + at] = lo;
    }
  }
};

// As attn_extend_kernel, for heads of 128 channels: a wavefront owns 32 columns and
// walks all steps of the workgroup's share, whose keys and values lie in LDS as
// bf16 tiles of 32 rows (uq_tile.h), copied a stage ahead.
// Codes in groups of 32 are made values on the way, two bf16 terms each (off by 2^-18
// of a value): both products then need neither scales nor offsets, and the work of
// that is shared by 128 columns.  With one group a head a scale and an offset a row
// cost less than the second terms' products, and the tiles hold the codes.
template <int FMT, int NG>
__global__ __launch_bounds__(256, 2) void attn_extend_wide_kernel(AttnExtendLaunch p, int target) {
  constexpr bool CODES = FMT != KV_BF16;
  constexpr int TERMS = CODES ? 2 : 1;              // of a key and of a value
  constexpr int STAGES = 2, STEPS = CODES ? 1 : 2;  // steps of a stage
  constexpr int TILE = 2 * TERMS * TILE16;          // a step's keys and values
  constexpr uint32_t ROW = FMT == KV_BF16 ? 256 : FMT == KV_U8 ? 128 : 64;
  __shared__ __attribute__((aligned(256))) u32x4a smem[STAGES][STEPS * TILE];
  const KvCache& c = p.c;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int G = p.H / c.H_kv;
  const int64_t b = workgroup();
  const int g = int(b % c.H_kv);
  Unit unit;
  if (!find<WIDE, false>(p, G, b / c.H_kv, target, unit)) return;
  const int s = unit.s;
  const Seq seq = seq_of(p, scalar(p.row_start, s), scalar(p.row_start, s + 1), scalar(p.lens, s));
  const Work<WIDE> work{p, G};
  const int tiles = work.tiles(seq), parts = uniform(unit.parts(work.steps(seq)));
  const int part = uniform(unit.at / tiles), tile = tiles - 1 - uniform(unit.at % tiles);  // the longest first
  const int len = capped(p, seq.len);
  const int base = seq.len < 0 ? -seq.m : std::max(seq.len - seq.m, -seq.m);
  const bool tree = p.mask != nullptr;

  // the lane's column, and what the workgroup's and the wavefront's see
  const int64_t idx = int64_t(tile) * WIDE + 32 * wave + (lane & 31);
  const int j = int(idx / G), head = g * G + int(idx % G);
  const int64_t row = j < seq.m && int64_t(seq.first) + j < p.T ? int64_t(seq.first) + j : -1;
  auto limits = [&](int64_t r, int j, int& end, int& low) {
    end = tree ? base : base + j + 1;
    const int64_t at = r >= 0 && p.pos ? p.pos[r] : int64_t(base) + j;
    low = p.window > 0 ? int(std::min<int64_t>(std::max<int64_t>(at - p.window + 1, 0), 0x7FFFFFFF)) : 0;
  };
  int end, low;
  limits(row, j, end, low);
  const int end_min = uniform(wave_min(row >= 0 ? end : 0x7FFFFFFF)), end_max = uniform(wave_max(row >= 0 ? end : 0));
  const int low_min = uniform(wave_min(row >= 0 ? low : 0x7FFFFFFF)), low_max = uniform(wave_max(row >= 0 ? low : 0));
  int all_end = 0, all_low = 0x7FFFFFFF;
  {
    __shared__ int ends[4], lows[4];
    if (lane == 0) {
      ends[wave] = end_max;
      lows[wave] = low_min;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      all_end = std::max(all_end, ends[w]);
      all_low = std::min(all_low, lows[w]);
    }
    all_end = uniform(all_end);
    all_low = uniform(all_low);
  }
  const int hi = tree ? len : std::min(len, all_end);
  const int lo = std::max(0, tree ? std::min(all_low, base) : all_low);
  const int n_sink = p.window > 0 ? (std::min(p.sinks, std::max(hi, 0)) + STEP - 1) / STEP : 0;
  const int u_lo = std::max(lo / STEP, n_sink);
  const int n_steps = n_sink + std::max(0, (std::max(hi, 0) + STEP - 1) / STEP - u_lo);
  const int i0 = uniform(int(int64_t(n_steps) * part / parts)), i1 = uniform(int(int64_t(n_steps) * (part + 1) / parts));
  auto step_at = [&](int i) { return i < n_sink ? i : u_lo + (i - n_sink); };

  const uint32_t page_bytes = uint32_t(c.H_kv) * uint32_t(c.page_len) * ROW;
  const uint32_t page_stats = uint32_t(c.H_kv) * uint32_t(c.page_len) * NG;
  const uint32_t head_bytes = uint32_t(g) * uint32_t(c.page_len) * ROW, head_stats = uint32_t(g) * uint32_t(c.page_len) * NG;
  const int32_t* pages = c.pages + int64_t(s) * c.max_pages;
  // where a step's two halves of 16 positions lie (of those on no page: page 0), and how many of them exist
  auto look_up = [&](int i, uint64_t (&at)[2], uint64_t (&st)[2], int (&nv)[2]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int pos = step_at(i) * STEP + 16 * t;
      const int page = i < i1 && pos < len ? scalar(pages, pos >> c.log_page) : -1;
      const bool is = page >= 0 && page < c.n_pages;
      const uint32_t pg = is ? uint32_t(page) : 0u, r = is ? uint32_t(pos & (c.page_len - 1)) : 0u;
      nv[t] = is ? std::min(16, len - pos) : 0;
      at[t] = uint64_t(pg) * page_bytes + (head_bytes + r * ROW);
      st[t] = uint64_t(pg) * page_stats + (head_stats + r);
    }
  };

  // queries, a negative scale's sign on them
  bf16x8a qf[8];
  {
    const uint16_t* q = p.Q + (row < 0 ? 0 : row) * p.ld_q + int64_t(head) * D + 8 * (lane >> 5);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      u32x4a v = row >= 0 ? *reinterpret_cast<const u32x4a*>(q + 16 * k) : u32x4a{0, 0, 0, 0};
      if (p.scale < 0.0f) v ^= 0x80008000u;
      qf[k] = __builtin_bit_cast(bf16x8a, v);
    }
  }
  const float cl = fabsf(p.scale) * LOG2E;  // scores to exponents of 2

  // copies of a bf16 cache straight into LDS, two blocks of 64 slots of every tile a wavefront
  uint32_t off[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int slot = (2 * wave + k) * 64 + lane, rho = slot >> 4;
    off[k] = uint32_t(perm32(rho) & 15) * ROW + uint32_t(((slot & 15) ^ swz(rho)) * 16);
  }
  uint64_t at[2], st[2];
  auto copy_stage = [&](int i, u32x4a* stage, int (&n)[STEPS][2]) {
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      look_up(i + t, at, st, n[t]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int blk = 2 * wave + k;  // rows of half blk / 4
        copy16(static_cast<const char*>(c.k) + at[blk >> 2], off[k], stage + t * TILE + blk * 64);
        copy16(static_cast<const char*>(c.v) + at[blk >> 2], off[k], stage + t * TILE + TILE16 + blk * 64);
      }
    }
  };
  Codes<CODES ? FMT : KV_U8> codes;

  f32x16a o[4] = {zero16(), zero16(), zero16(), zero16()};
  // weights count in 2^-24 against the running maximum (see attn_decode.hip): m is 24 above it
  constexpr float DOWN = 24.0f;
  float m = LOWEST, l = 0.0f;

  const LaneTile frags(smem[0], lane);
  // products of one step out of tile tk, at `bytes` of the stages, nvt of whose positions exist
  auto step = [&](const u32x4a* tk, uint32_t stage, uint32_t bytes, int t0, const int (&nvt)[2]) {
    const u32x4a* tv = tk + TERMS * TILE16;
    const LaneTile f = frags.at(stage);
    f32x16a x = zero16();
#pragma unroll
    for (int term = 0; term < TERMS; ++term)
#pragma unroll
      for (int k = 0; k < 8; ++k) x = mfma(f.row(k, bytes + term * TILE16 * 16), qf[k], x);
    const bool cut = nvt[0] + nvt[1] < STEP || t0 + STEP > end_min || (t0 < low_max && t0 + STEP > p.sinks);
    uint32_t seen = 0;  // bit r: slot r
    if (cut) {
      uint32_t drafts = 0;
      if (tree && t0 + STEP > base && row >= 0) drafts = mask_bits(p.mask + row * p.words, p.words, t0 - base);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int in = slot_row(r, lane), at = t0 + in;
        const bool ok = at < end ? (at >= low || (p.window > 0 && at < p.sinks)) : (at >= base && (drafts >> in & 1));
        seen |= ok && (in & 15) < nvt[r >> 3] ? 1u << r : 0u;
        x[r] = seen >> r & 1 ? x[r] : -__builtin_inff();
      }
    }
    float mx = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
    mx = max2(mx) * cl;
    if (__any(mx > m - DOWN + SLACK)) {
      const float m1 = mx > m - DOWN + SLACK ? mx + DOWN : m;
      const float f = exp2a(m - m1);
      m = m1;
      l *= f;
#pragma unroll
      for (int db = 0; db < 4; ++db) o[db] *= f;
    }
    float w[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r] = exp2a(__builtin_fmaf(x[r], cl, -m));
    bool wild_values = false;
    if (cut) {
#pragma unroll
      for (int r = 0; r < 16; ++r) w[r] = seen >> r & 1 ? w[r] : 0.0f;
      // values that are not finite, which a weight of 0 does not take out of a product
      bool any = false;
      for (int k = 0; k < TILE16 / 64; ++k) {
        const u32x4a v = tv[k * 64 + lane];
        any |= wild(v.x) || wild(v.y) || wild(v.z) || wild(v.w);
      }
      wild_values = __any(any);
    }
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += w[r];
    l += sum;
    if (wild_values) {
      // one position after the other, those with a weight only
#pragma unroll 1
      for (int pos = 0; pos < STEP; ++pos) {
        // held by lane half (pos / 8) % 2 in slot 8 (pos / 16) + pos % 8
        float z = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (r == 8 * (pos >> 4) + (pos & 7)) z = __shfl(w[r], (lane & 31) + 32 * (pos >> 3 & 1));
        z = float(__bf16(z));
        const int rho = perm32(pos);
        const uint16_t* vrow = reinterpret_cast<const uint16_t*>(tv + rho * 16);
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int ch = 32 * db + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
            const int at = ((ch >> 3) ^ swz(rho)) * 8 + (ch & 7);
            float v = bf16_to_f32(vrow[at]);
            if constexpr (TERMS == 2) v += bf16_to_f32(vrow[TILE16 * 8 + at]);
            if (z != 0.0f) o[db][r] += z * v;
          }
      }
      return;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x8a pb = pack_half(w, h);
#pragma unroll
      for (int term = 0; term < TERMS; ++term)
#pragma unroll
        for (int db = 0; db < 4; ++db) o[db] = mfma(f.col(db, h, bytes + (TERMS + term) * TILE16 * 16), pb, o[db]);
    }
  };

  int nv[STEPS][2], nv_next[STEPS][2], cur = 0;
  if constexpr (CODES) {
    look_up(i0, at, st, nv[0]);
    codes.load(c, at, st, nv[0]);
    codes.store(smem[0]);
    look_up(i0 + 1, at, st, nv_next[0]);
    codes.load(c, at, st, nv_next[0]);
    __syncthreads();
  } else {
    copy_stage(i0, smem[0], nv);
  }
  for (int i = i0; i < i1; i += STEPS, cur ^= 1) {
    if constexpr (CODES) {
      step(smem[cur], cur * uint32_t(sizeof(smem[0])), 0, step_at(i) * STEP, nv[0]);
      codes.store(smem[cur ^ 1]);
      nv[0][0] = nv_next[0][0];
      nv[0][1] = nv_next[0][1];
      look_up(i + 2, at, st, nv_next[0]);
      codes.load(c, at, st, nv_next[0]);
      __syncthreads();
    } else {
      vm_wait<0>();
      lds_wait_barrier();
      copy_stage(i + STEPS, smem[cur ^ 1], nv_next);
#pragma unroll
      for (int t = 0; t < STEPS; ++t)
        if (i + t < i1)
          step(smem[cur] + t * TILE, cur * uint32_t(sizeof(smem[0])), t * TILE * 16, step_at(i + t) * STEP, nv[t]);
#pragma unroll
      for (int t = 0; t < STEPS; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k) nv[t][k] = nv_next[t][k];
    }
  }
  if constexpr (!CODES) vm_wait<0>();  // no copy is on its way when the workgroup ends

  l += other_half(l);
  if (row < 0) return;
  if (parts == 1) {
    const float inv = 1.0f / l;
    uint16_t* out = p.O + row * p.ld_o + int64_t(head) * D;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const uint32_t a = pack_bf16x2(o[db][4 * g4] * inv, o[db][4 * g4 + 1] * inv);
        const uint32_t e = pack_bf16x2(o[db][4 * g4 + 2] * inv, o[db][4 * g4 + 3] * inv);
        // no weight at all: 0
        *reinterpret_cast<u32x2a*>(out + 32 * db + 8 * g4 + 4 * (lane >> 5)) = l == 0.0f ? u32x2a{0, 0} : u32x2a{a, e};
      }
    if (lane < 32 && p.lse) p.lse[row * p.H + head] = l == 0.0f ? -__builtin_inff() : m + __builtin_amdgcn_logf(l);
    return;
  }
  const int64_t slot = int64_t(unit.slot) + unit.at;
  if (slot >= int64_t(target)) return;
  float* out = part_of<WIDE, D>(p, slot, g, 32 * wave + (lane & 31));
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      *reinterpret_cast<float4*>(out + 4 + 32 * db + 8 * g4 + 4 * (lane >> 5)) =
          make_float4(o[db][4 * g4], o[db][4 * g4 + 1], o[db][4 * g4 + 2], o[db][4 * g4 + 3]);
  if (lane < 32) *reinterpret_cast<float2*>(out) = make_float2(m, l);
}

// Joins the shares of a tile's columns: D / 4 lanes a share of a column, PAR
// shares of it at a time, four of each in flight; 256 / (PAR D / 4) columns.
template <int D, int COLS, int PAR>
__global__ __launch_bounds__(256) void attn_extend_join_kernel(AttnExtendLaunch p, int target, float back) {
  constexpr int LANES = D / 4, ROWS = 256 / LANES / PAR, GROUPS = COLS / ROWS;
  const int G = p.H / p.c.H_kv;
  const int64_t b = workgroup();
  const int g = int(b % p.c.H_kv), group = int(b / p.c.H_kv % GROUPS);
  Unit unit;
  if (!find<COLS, true>(p, G, b / p.c.H_kv / GROUPS, target, unit)) return;
  const int s = unit.s;
  const Seq seq = seq_of(p, scalar(p.row_start, s), scalar(p.row_start, s + 1), scalar(p.lens, s));
  const Work<COLS> work{p, G};
  const int tiles = work.tiles(seq), n = unit.parts(work.steps(seq));
  const int lane = threadIdx.x % LANES, rank = threadIdx.x / LANES % PAR, col = group * ROWS + threadIdx.x / LANES / PAR;
  const int tile = unit.at;
  const int64_t idx = int64_t(tile) * COLS + col;
  const int64_t r = int64_t(seq.first) + idx / G;
  const bool real = idx / G < seq.m && r < p.T && int64_t(unit.slot) + int64_t(n) * tiles <= int64_t(target);
  float m = LOWEST, t = 0.0f;
  f32x4d a = {};
  if (real) {
    for (int k = rank; k < n; k += 4 * PAR) {
      float2 ml[4];
      f32x4d o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = std::min(k + i * PAR, n - 1);
        const float* part = part_of<COLS, D>(p, int64_t(unit.slot) + int64_t(j) * tiles + (tiles - 1 - tile), g, col);
        ml[i] = *reinterpret_cast<const float2*>(part);
        o[i] = *reinterpret_cast<const f32x4d*>(part + 4 + 4 * lane);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (k + i * PAR >= n) break;
        const float m1 = fmaxf(m, ml[i].x);
        const float f0 = __builtin_amdgcn_exp2f(m - m1), f1 = __builtin_amdgcn_exp2f(ml[i].x - m1);
        m = m1;
        t = t * f0 + ml[i].y * f1;
        a = a * f0 + o[i] * f1;
      }
    }
  }
  if constexpr (PAR > 1) {
    __shared__ f32x4d so[256];
    __shared__ float sm[256 / LANES], st[256 / LANES];
    so[threadIdx.x] = a;
    if (lane == 0) {
      sm[threadIdx.x / LANES] = m;
      st[threadIdx.x / LANES] = t;
    }
    __syncthreads();
    if (rank) return;
    const int first = threadIdx.x / LANES;
    float top = sm[first];
#pragma unroll
    for (int k = 1; k < PAR; ++k) top = fmaxf(top, sm[first + k]);
    t = 0.0f;
    a = f32x4d{};
#pragma unroll
    for (int k = 0; k < PAR; ++k) {
      const float f = __builtin_amdgcn_exp2f(sm[first + k] - top);
      t += f * st[first + k];
      a += f * so[(first + k) * LANES + lane];
    }
    m = top;
  }
  if (!real) return;
  const int hd = g * G + int(idx % G);
  const float inv = back / t;
  *reinterpret_cast<uint2*>(p.O + r * p.ld_o + int64_t(hd) * D + 4 * lane) =
      t == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(a[0] * inv, a[1] * inv), pack_bf16x2(a[2] * inv, a[3] * inv));
  if (lane == 0 && p.lse) p.lse[r * p.H + hd] = t == 0.0f ? -__builtin_inff() : m + __builtin_amdgcn_logf(t);
}

// Columns of a workgroup, for those that a sequence has on average: 16, 32, and of heads of 128 channels WIDE
// (us, 24 sequences of 8192 positions, 8 key/value heads, with 16 | 32 | 128 columns):
//   32 columns:  bf16 185 | 171 | 225,  u8 113 | 103 | -,    u8 in groups of 32 144 | 361 | 296
//   64 columns:  bf16 264 | 185 | 212,  u8 178 | 124 | -,    u8 in groups of 32 235 | 552 | 315
//   128 columns: bf16 474 | 275 | 229,  u8 317 | 202 | 276,  u8 in groups of 32 423 | 957 | 338
// and of heads of 64 channels, with 16 | 32:
//   32 columns:  bf16 94 | 87,    u8 55 | 57,    u8 in groups of 32 65 | 65
//   128 columns: bf16 274 | 155,  u8 174 | 147,  u8 in groups of 32 213 | 178
// One sequence of 32768 positions goes alike; batches too small to fill the GPU lose up to 17 us by the larger tiles
// (4 sequences of 4096 positions, 2 heads, 128 columns: bf16 26 | 28 | 34, u8 22 | 26 | -, in groups of 32 25 | - | 42).
// Two column tiles and the statistics of four groups do not fit into the registers.
enum Kind { PLAIN, ONE_GROUP, GROUPS };
constexpr Kind kind_of(int fmt, int ng) { return fmt == KV_BF16 ? PLAIN : ng == 1 ? ONE_GROUP : GROUPS; }
int columns_of(int64_t T, int64_t n_seq, int H, int H_kv, int d, Kind f) {
  const int64_t cols = (T + n_seq - 1) / n_seq * (H / H_kv);
  if (cols <= 16) return 16;
  if (d != 128 || f == ONE_GROUP) return 32;
  return cols > 64 ? WIDE : f == PLAIN ? 32 : 16;
}
// Tiles of one key/value head, if no row is padding; workgroups for them and as many shares (or numbers, find_whole).
int64_t tiles_of(int64_t T, int H, int H_kv, int cols) { return T * (H / H_kv) / cols; }
int64_t units_of(const AttnExtendLaunch& p, int cols, int target) {
  return tiles_of(p.T, p.H, p.c.H_kv, cols) + (target ? std::min(p.T, p.c.n_seq) + target : p.c.n_seq);
}
// Whether a tile can be cut at all: two shares of a key/value head have to have a place, and steps enough.
bool cuttable(int H_kv, int64_t max_pages, int page_len) {
  return 2 * CUS / H_kv >= 2 && max_pages * page_len > MIN_STEPS * STEP;
}
// Shares of one key/value head that are wanted (0: no tile is cut; else two or more).  The GPU holds two workgroups a
// CU; between a quarter of those and all, two rounds of shares even out what rounding shares of whole steps leaves
// (24 x 32 rows of 8192 positions at 8 bits, 1.5 tiles a place: 245 us with one round, 250 with two).  With more tiles
// than places only a tile of twice the mean and more is cut, which costs equal sequences the join (1 x 2048 rows 85 ->
// 92 us) and saves unequal ones more (96 x 8 rows, one sequence of 32768 positions and 95 of 1024: 470 -> 134 us).
int target_of(int64_t T, int64_t n_seq, int H, int H_kv, int cols, int64_t max_pages, int page_len) {
  const int64_t holds = 2 * CUS / H_kv, tiles = std::max(tiles_of(T, H, H_kv, cols), std::min(T, n_seq));
  if (!cuttable(H_kv, max_pages, page_len) || tiles >= 4 * holds) return 0;
  return int(4 * tiles <= holds || tiles >= holds ? holds : 2 * holds);
}

// Where sequences have more than 64 columns on average, those with few have a launch of the smaller tiles to
// themselves (single tokens beside a prompt), up to few_of columns, in so many shares.  One prompt of 512 rows and
// single tokens, 8192 positions each, 32 heads over 8: 31 tokens in bf16 366 -> 334 us, of 8 bits in groups of 32
// 632 -> 367; 7 tokens 198 -> 165 and 325 -> 222.  Sequences alike pay the empty launches (8 x 128 rows 225 -> 230 us,
// 359 -> 370), so that fewer than four go without.
int few_of(Kind f) { return f == PLAIN ? 16 : 64; }
bool few_apart(int64_t n_seq, int H_kv, int64_t max_pages, int page_len) {
  return n_seq >= 4 && cuttable(H_kv, max_pages, page_len);
}
// (Not cut above 1024 sequences, which every workgroup would add up: 1024 x 70 rows over 400 positions of 8 heads 880
// us, 1025 so 635; 128 prompts of 700 rows beside 896 single tokens over 2000 positions 2530, one more so 2467.)
int target_of_few(int64_t n_seq, int H_kv, int64_t max_pages, int page_len) {
  return few_apart(n_seq, H_kv, max_pages, page_len) && n_seq <= 1024 ? 2 * CUS / H_kv : 0;
}

template <int D, int COLS>
hipError_t launch_join(const AttnExtendLaunch& p, int target, float back, hipStream_t st) {
  constexpr int LANES = D / 4;
  const int64_t tiles = std::min<int64_t>(tiles_of(p.T, p.H, p.c.H_kv, COLS) + std::min(p.T, p.c.n_seq), target / 2);
  if (p.T * p.H <= 2048)
    attn_extend_join_kernel<D, COLS, 256 / LANES><<<grid_of(tiles * p.c.H_kv * COLS), 256, 0, st>>>(p, target, back);
  else
    attn_extend_join_kernel<D, COLS, 1><<<grid_of(tiles * p.c.H_kv * COLS * LANES / 256), 256, 0, st>>>(p, target, back);
  return hipGetLastError();
}

template <int FMT, int D, int NG>
hipError_t launch_form(const AttnExtendLaunch& p, hipStream_t st) {
  constexpr Kind KIND = kind_of(FMT, NG);
  const int H_kv = p.c.H_kv, cols = columns_of(p.T, p.c.n_seq, p.H, H_kv, D, KIND);
  const int target = target_of(p.T, p.c.n_seq, p.H, H_kv, cols, p.c.max_pages, p.c.page_len);
  const dim3 grid = grid_of(units_of(p, cols, target) * H_kv);
  const float back = FMT == KV_BF16 ? BF16_BACK : 1.0f;
  if constexpr (D == 128 && KIND != ONE_GROUP) {
    if (cols == WIDE) {
      AttnExtendLaunch many = p, few = p;
      const bool apart = few_apart(p.c.n_seq, H_kv, p.c.max_pages, p.c.page_len);
      if (apart) many.from_cols = (few.to_cols = few_of(KIND)) + 1;
      attn_extend_wide_kernel<FMT, NG><<<grid, 256, 0, st>>>(many, target);
      if (hipError_t e = hipGetLastError()) return e;
      if (apart) {
        const int few_target = target_of_few(p.c.n_seq, H_kv, p.c.max_pages, p.c.page_len);
        const int64_t n = (few_target ? std::min(p.T, p.c.n_seq) : p.c.n_seq) * (few_of(KIND) / 16) + few_target;
        few.ws = p.ws + size_t(target) * size_t(H_kv) * WIDE * (D + 4);
        attn_extend_kernel<FMT, D, NG, 1><<<grid_of(n * H_kv), 256, 0, st>>>(few, few_target);
        if (hipError_t e = hipGetLastError()) return e;
        if (few_target) {
          if (hipError_t e = launch_join<D, 16>(few, few_target, back, st)) return e;
        }
      }
      return target ? launch_join<D, WIDE>(many, target, 1.0f, st) : hipSuccess;
    }
  }
  if constexpr (D == 64 || KIND != GROUPS) {
    if (cols == 32) {
      attn_extend_kernel<FMT, D, NG, 2><<<grid, 256, 0, st>>>(p, target);
      if (hipError_t e = hipGetLastError()) return e;
      return target ? launch_join<D, 32>(p, target, back, st) : hipSuccess;
    }
  }
  attn_extend_kernel<FMT, D, NG, 1><<<grid, 256, 0, st>>>(p, target);
  if (hipError_t e = hipGetLastError()) return e;
  return target ? launch_join<D, 16>(p, target, back, st) : hipSuccess;
}

template <int D>
hipError_t launch_d(const AttnExtendLaunch& p, hipStream_t st) {
  const bool one = p.c.group == D;
  if (p.c.format == KV_BF16) return launch_form<KV_BF16, D, 1>(p, st);
  if (p.c.format == KV_U8) return one ? launch_form<KV_U8, D, 1>(p, st) : launch_form<KV_U8, D, D / 32>(p, st);
  return one ? launch_form<KV_U4, D, 1>(p, st) : launch_form<KV_U4, D, D / 32>(p, st);
}

}  // namespace

size_t attn_extend_ws(int64_t T, int64_t n_seq, int H, int H_kv, int d, int64_t max_pages, int page_len) {
  size_t most = 0;  // of all formats
  for (const Kind f : {PLAIN, ONE_GROUP, GROUPS}) {
    const int cols = columns_of(T, n_seq, H, H_kv, d, f);
    const size_t few = cols == WIDE ? size_t(target_of_few(n_seq, H_kv, max_pages, page_len)) * 16 : 0;
    most = std::max(most, size_t(target_of(T, n_seq, H, H_kv, cols, max_pages, page_len)) * size_t(cols) + few);
  }
  return most * size_t(H_kv) * size_t(d + 4);
}

hipError_t launch_attn_extend(AttnExtendLaunch p, hipStream_t st) {
  p.from_cols = 0;
  p.to_cols = INT64_MAX;
  return p.c.d == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace uq
