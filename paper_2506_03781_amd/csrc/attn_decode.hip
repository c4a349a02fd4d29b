// Attention of one new token per sequence over the paged key/value cache
// (uniquan_attn_decode); layout, formulas and errors in uniquan.h.
//
// Split.  A workgroup of four wavefronts takes one key/value head, up to 16 of
// its query heads and an equal share of all sequences' positions, as many
// workgroups as the GPU holds at once: positions count in blocks of 128 (each
// wavefront a step of 32), and every sequence costs a block more, its end.  A
// share is a run of blocks over one or several sequences (Share); its part of
// one sequence is a chunk.  The wavefronts' steps of a chunk, each with a
// running maximum and sum, are joined in LDS; a sequence that lies in one
// share is finished there, the chunks of the others are joined by
// attn_join_kernel.
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
// Statistics.  The scale and offset of a position belong to a row of S^T and
// are wanted in every column; the matrix cores spread them: a lane loads the
// (scale, offset) pair of position l % 16 as it stands (two bf16 values), and a
// product with a column of constants gives the scale, the offset times sum q
// or the value of the codes' middle in the layout of S^T
// (v_mfma_f32_16x16x16_bf16, k = 4 (l / 16) .. + 4: the pair is slots 0 and 1
// of the lane's four, and with several groups lane / 16 takes one each; sum q
// in three bf16 terms against three copies of the pair, 32 deep).
//
// Precision.  Scores are fp32 sums of exact products.  A weight p (times the
// group's scale for codes) enters the second product as two bf16 terms, the
// truncated value and the truncated rest: with up to 8 heads the rest stands in
// the columns 8..15, which costs nothing, above that in a second product.  The
// rest is below 2^-7 of p and its truncation takes less than 2^-15 off, 2^-17 on
// average, so p 2^-17 is added to it first: what the terms miss lies between
// -2^-17 and 2^-15 - 2^-17 of p and does not add up over a row.  And the rest of
// a weight is above 0 as the weight is, so that an infinite value stays infinite
// (0 times it is NaN) down to weights of 2^-92.  Values of a bf16 cache meet
// weights 2^-24 times their size: of at most 2^-16, so that a row of 2^16 of the
// largest bf16 numbers stays in fp32's range until it is divided by the weights'
// sum, while a rounding among the smallest fp32 numbers takes 2^-126 off the
// output.  Every step takes the codes' middle away again with the same bf16
// terms (a product with a constant), and the exact weights carry the middle's
// value: what truncation takes off the terms then scales values around zero,
// not their offset, which in a long row is hundreds of times the output.
//
// Codes as bf16.  A code c enters as c 2^-133: its bits at the foot of a bf16
// word, which is that number below 128 (subnormal) and above (exponent 1)
// alike, and exact.  An 8-bit code takes half a byte permutation; of a byte
// with two 4-bit codes one AND takes the lower, another the upper as 16 c, for
// which its query channels are 16 times smaller and its output channels are
// divided by 16.  (Fed as 128 + c the codes need a shift and an AND-OR each and
// the 128 taken away again: as fast, but scores of short rows were off by up to
// 6e-6 of their size, now 3e-7.)  The queries of a head are scaled by a power
// of two to a largest magnitude in [2^120, 2^121) and the scales by 2^64
// against it.  So scales of keys may reach 2^60 and those of values 2^55 (their
// weights 2^8), offsets of either 2^60; sums of values stand 2^-69 times their
// size in fp32, whose roundings are 2^-150 at the least: 2^-81 of the output.
//
// Bound and measured (the kernel alone; a sequence split over shares adds the
// join, 4 to 8 us, a launch and two loads that wait on each other).  bf16 and
// 8-bit caches by memory: 64 sequences of up to 16384 positions, 64 heads on 8,
// 1.96 GB in 337 us, 5.8 TB/s; 48 of up to 8192 at 8 bits 391 MB in 75 us, 5.2
// TB/s; 4 of 2048, 32 heads, 134 MB in 25.7 us, 5.2 TB/s.  4-bit caches read a
// quarter of the bytes with the same number of loads: 100001 positions in groups
// of 32 128 MB in 33.4 us, 3.8 TB/s, vector instructions in 57% of the cycles,
// matrix ones in 24%.  One sequence of 100 positions 5.7 us: a launch and the
// loads of its length, its page and its rows, one after the other.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "uq_attend.h"
#include "uq_device.h"
#include "uq_kv.h"
#include "uq_launch.h"

namespace uq {

namespace {

constexpr int BLOCK = WAVES * STEP;         // positions of a workgroup's round
// Least blocks of a share, ends counted (with 1, 2 and 4: one sequence of 8192 positions, 64 heads on 8, 16.5,
// 14.4 and 15.0 us; 4 of 2048 15.4, 16.1 and 14.6; 4 of up to 1000 at 8 bits 12.8, 12.9 and 14.8).
constexpr int MIN_COST = 2;

// ---------------------------------------------------------------------------
// which positions a workgroup takes
// ---------------------------------------------------------------------------
__device__ __forceinline__ int capped(const AttnDecodeLaunch& p, int len) {
  const int64_t cap = p.c.max_pages << p.c.log_page;
  return len < 0 ? 0 : int(len < cap ? len : cap);
}

__device__ __forceinline__ int blocks_of(int len) { return (len + BLOCK - 1) / BLOCK; }

// Share `at` of `want`: [a, b) of the sequences' costs laid end to end, from
// sequence s on, whose cost begins at `begin`.
struct Share {
  int a, b;
  int s, begin;
  int total;  // cost of all sequences
};

__device__ __forceinline__ int parts_of(int total, int want) { return std::min(want, std::max(1, total / MIN_COST)); }

// Every wavefront works it out by itself: its lanes add up runs of the
// sequences, then the run that holds `a` is searched.  With little in all,
// only the first shares get something, MIN_COST at least.
__device__ __forceinline__ Share share_of(const AttnDecodeLaunch& p, int at, int want) {
  if (want == 1) return Share{0, 0x7FFFFFFF, 0, 0, 0};
  const int lane = threadIdx.x & 63;
  const int n = int(p.c.n_seq);
  const int per = (n + 63) / 64;
  auto cost = [&](int j) { return j < n ? blocks_of(capped(p, p.lens[j])) + 1 : 0; };
  int mine = 0;
  for (int j = lane * per; j < lane * per + per; ++j) mine += cost(j);
  int upto = wave_scan(mine);
  const int total = __builtin_amdgcn_readlane(upto, 63);
  const int parts = parts_of(total, want);
  if (at >= parts) return Share{0, 0, 0, 0, total};
  const int q = total / parts, r = total % parts;
  Share h;
  h.total = total;
  h.a = at * q + at * r / parts;
  h.b = (at + 1) * q + (at + 1) * r / parts;
  // the run that holds a (it is below total), then the sequence in it, 64 at a time
  int in = __builtin_ctzll(__ballot(upto > h.a) | 1ull << 63);
  h.s = in * per;
  h.begin = __builtin_amdgcn_readlane(upto - mine, in);
  if (per == 1) return h;
  for (const int end = h.s + per; h.s < end; h.s += 64) {
    mine = h.s + lane < end ? cost(h.s + lane) : 0;
    upto = wave_scan(mine) + h.begin;
    const uint64_t past = __ballot(upto > h.a);
    if (past) {
      in = __builtin_ctzll(past);
      h.s += in;
      h.begin = __builtin_amdgcn_readlane(upto - mine, in);
      return h;
    }
    h.begin = __builtin_amdgcn_readlane(upto, 63);
  }
  return Share{0, 0, 0, 0, total};
}

// A share's part of one sequence: blocks [b0, b1); the sequence's first and
// last lie in it where it opens and closes.
struct Chunk {
  int64_t s;
  int len, b0, b1, end;  // end: of the sequence's cost
  bool opens, closes;
};

// The share's next chunk after c (the first for c.s = share.s - 1, c.end =
// share.begin); false: none.  A sequence without positions is a chunk too,
// where it opens.
__device__ __forceinline__ bool next_chunk(const AttnDecodeLaunch& p, const Share& h, Chunk& c) {
  while (c.end < h.b && ++c.s < p.c.n_seq) {
    const int begin = c.end;
    c.len = capped(p, scalar(p.lens, c.s));
    const int blocks = blocks_of(c.len);
    c.end = begin + blocks + 1;
    c.b0 = std::max(h.a - begin, 0);
    c.b1 = std::min(h.b - begin, blocks);
    c.opens = begin >= h.a;
    c.closes = begin + blocks <= h.b;
    if (c.b0 < c.b1 || (blocks == 0 && c.opens)) return true;
  }
  return false;
}

// The workspace: notes of the sequences that lie in several shares, one a
// sequence, or one a share (the sequence that begins in it) where there are
// fewer shares, so that no more joins are launched than are wanted (4096
// sequences of 128 positions, 32 heads on 8, in 96 shares: 353 us with one a
// sequence, 288 with one a share); then two chunks a share, of the sequence that
// came into it and of the one that goes out, H rows each of (maximum, sum, -, -,
// D values) against that maximum.
struct Note {
  int share, s;  // the first share
  int last;      // the cost of its last block, -1: the sequence lies in one share
  int total;     // Share's
};
__host__ __device__ __forceinline__ int64_t notes_of(const KvCache& c, int want) { return c.n_seq < want ? c.n_seq : want; }
__device__ __forceinline__ Note* notes(const AttnDecodeLaunch& p) { return reinterpret_cast<Note*>(p.ws); }
__device__ __forceinline__ float* chunk(const AttnDecodeLaunch& p, int want, int share, bool opens, int64_t head, int D) {
  return p.ws + notes_of(p.c, want) * 4 + ((2 * int64_t(share) + opens) * p.H + head) * (D + 4);
}

// ---------------------------------------------------------------------------
// one chunk
// ---------------------------------------------------------------------------
// Workgroups a CU holds (their registers are bounded to that): the most for
// which nothing is spilled in the loop, measured one less and one more.  bf16
// with 128 channels has room for three and loses by it (7B block, 4 x 2048:
// 30.0 us against 31.2; 64 x up to 16384 352 against 355); 4-bit groups of 32 46
// us with three against 40 (100001 positions), 8-bit ones 138 against 90 (48
// ragged sequences) and, with 64 channels, 55 with four against 50.
template <int FMT, int D, int NG>
constexpr int kResident = D == 64 ? (FMT == KV_U8 && NG > 1 ? 3 : 4) : FMT == KV_BF16 || NG > 1 ? 2 : 3;

// WIDE: 16 query heads a workgroup, else 8 with the weights' rests in the upper columns.
template <int FMT, int D, int NG, bool WIDE>
__global__ __launch_bounds__(256, (kResident<FMT, D, NG>)) void attn_decode_kernel(AttnDecodeLaunch p, int want,
                                                                                   int rtiles) {
  using F = Form<FMT, D>;
  constexpr int HEADS = WIDE ? 16 : 8;
  constexpr bool CODES = FMT != KV_BF16;
  constexpr float MID = FMT == KV_U8 ? 128.0f : 8.0f;
  constexpr float VSCALE = 0x1p64f;  // on the scales
  constexpr float VBACK = 0x1p69f;   // 2^133 / VSCALE
  // 4-bit codes of the odd channel tiles come 16-fold
  auto sixteenfold = [](int k) { return FMT == KV_U4 && k % 2 == 1; };
  constexpr int LD = D + 4;
  __shared__ __attribute__((aligned(16))) float so[WAVES][16][LD];
  __shared__ float sm[WAVES][16], ss[WAVES][16];
  const KvCache& c = p.c;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int col = lane & 15, grp = lane >> 4;
  // consecutive workgroups go to the 8 XCDs in turn: the row tiles that read one head's cache 8 apart
  const unsigned b = blockIdx.x;
  const unsigned unit = b / (8 * rtiles) * 8 + b % 8;
  const int rt = int(b / 8 % rtiles);
  const int at = int(unit / c.H_kv), g = int(unit % c.H_kv);
  if (at >= want) return;
  const Share share = share_of(p, at, want);
  const bool noting = p.ws && g == 0 && rt == 0 && threadIdx.x == 0, by_seq = p.c.n_seq <= want;
  if (noting && !by_seq) notes(p)[at].last = -1;
  const int grp_heads = p.H / c.H_kv;
  const int h_in = rt * HEADS + (col & (HEADS - 1));  // head within its key/value head's group
  const bool rest = !WIDE && col >= 8;
  const uint32_t cut = rest ? 0xFFFF0000u : 0u;
  const float grown = rest ? MORE : 1.0f;

  const uint32_t page_bytes = uint32_t(c.H_kv) * uint32_t(c.page_len) * F::ROW;
  const uint32_t page_stats = uint32_t(c.H_kv) * uint32_t(c.page_len) * NG;
  const uint32_t head_bytes = uint32_t(g) * uint32_t(c.page_len) * F::ROW;
  // the lane's word of statistics in a tile: position l % 16 of group l / 16
  const uint32_t lane_stat = (uint32_t(g) * NG + uint32_t(grp % NG)) * uint32_t(c.page_len) + col;
  // columns of constants that take a group's scale (times VSCALE), and its middle's value, out of the pairs
  uint32_t pick[NG], mids[NG];
#pragma unroll
  for (int e = 0; e < NG; ++e) {
    pick[e] = grp == e ? pair(VSCALE, 0.0f) : 0u;
    mids[e] = grp == e ? pair(MID, 1.0f) : 0u;
  }

  // The loads run a step ahead of the products, over the chunks' ends: the next
  // step's keys are asked for when this step's scores are done, its values when
  // they are used up, in the same registers; its pages were looked up before.
  // Behind the last step, and for a tile on no page, the loads go to page 0.
  struct Ahead {
    Chunk c;
    bool is;
    int u, u1, page[2];
    uint64_t place[2], stat[2];
    int nv[2];  // positions of each tile that take part
  } next;
  uint32_t kw[2][F::KW], vw[8][F::VW], kst[2], vst[2];
  auto look_up = [&] {
    const int32_t* pages = c.pages + next.c.s * c.max_pages;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int base = next.u * STEP + 16 * t;
      next.page[t] = next.is && base < next.c.len ? scalar(pages, base >> c.log_page) : -1;
    }
  };
  auto open_chunk = [&](bool is) {  // next.c, if it is one, or the first after it with positions
    while (is && next.c.b0 >= next.c.b1) is = next_chunk(p, share, next.c);
    next.is = is;
    next.u = next.c.b0 * WAVES + wave;
    next.u1 = next.c.b1 * WAVES;
  };
  auto load_keys = [&] {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int base = next.u * STEP + 16 * t;
      const bool is = next.page[t] >= 0 && next.page[t] < c.n_pages;
      const uint32_t pg = is ? uint32_t(next.page[t]) : 0u;
      const uint32_t r = is ? uint32_t(base & (c.page_len - 1)) : 0u;
      next.nv[t] = is ? std::min(16, next.c.len - base) : 0;
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
    next.u += WAVES;
    if (next.u >= next.u1) open_chunk(next_chunk(p, share, next.c));
    look_up();
  };
  // A chunk's queries are asked for while the chunk before is joined (65536 sequences of 64 positions 763 us
  // against 808), the first chunk's before any keys (100001 positions at 4 bits 37.9 us against 38.5).
  u32x4d q[F::NC];
  Chunk ch{int64_t(share.s) - 1, 0, 0, 0, share.begin, false, false};
  auto load_queries = [&] {
    const uint16_t* row = p.Q + ch.s * p.ld_q + (int64_t(g) * grp_heads + h_in) * D + 8 * grp;
#pragma unroll
    for (int k = 0; k < F::NC; ++k)
      q[k] = h_in < grp_heads ? *reinterpret_cast<const u32x4d*>(row + 32 * k) : u32x4d{0, 0, 0, 0};
  };
  bool more = next_chunk(p, share, ch);
  if (more) load_queries();
  next.c = ch;
  open_chunk(more);
  look_up();
  load_keys();
  int nv[2] = {next.nv[0], next.nv[1]};
  load_values();

  while (more) {
    const int64_t s = ch.s;
    const bool opens = ch.opens, closes = ch.closes;
    if (noting && opens && (by_seq || !closes)) notes(p)[by_seq ? s : at] = {at, int(s), closes ? -1 : ch.end - 2, share.total};

    // queries (a negative scale's sign put on them), and for codes their sums over each group of channels
    float cl = fabsf(p.scale) * LOG2E_D;  // scores to exponents of 2
    u32x4d qs = {};  // the sum of the lane's group in three bf16 terms, against (scale, offset)
    {
      if (p.scale < 0.0f) {
#pragma unroll
        for (int k = 0; k < F::NC; ++k) q[k] ^= 0x80008000u;
      }
      if constexpr (CODES) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < F::NC; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = std::max(top, std::max(q[k][i] << 16 & 0x7FFF0000u, q[k][i] & 0x7FFF0000u));
        const int ex = int(__float_as_uint(max4(__uint_as_float(top))) >> 23) - 127;
        const float up = ldexpf(1.0f, 120 - std::max(ex, -7));
        cl = cl * ldexpf(1.0f, 13 - 64 + std::max(ex, -7));  // 2^133 over the queries' power and the scales'
#pragma unroll
        for (int k = 0; k < F::NC; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            q[k][i] = pair(__uint_as_float(q[k][i] << 16) * up, __uint_as_float(q[k][i] & 0xFFFF0000u) * up);
        float mine = 0.0f;
#pragma unroll
        for (int e = 0; e < NG; ++e) {
          float t = 0.0f;
#pragma unroll
          for (int k = e * F::NC / NG; k < (e + 1) * F::NC / NG; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              t += __uint_as_float(q[k][i] << 16) * 0x1p-69f + __uint_as_float(q[k][i] & 0xFFFF0000u) * 0x1p-69f;
          t = sum4(t);
          if (grp == e) mine = t;
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const float h = __uint_as_float(__float_as_uint(mine) & 0xFFFF0000u);
          qs[i] = pair(0.0f, h);
          mine -= h;
        }
        if constexpr (FMT == KV_U4) {
#pragma unroll
          for (int k = 0; k < F::NC; ++k)
#pragma unroll
            for (int i = 1; i < 4; i += 2)
              q[k][i] = pair(__uint_as_float(q[k][i] << 16) * 0x1p-4f, __uint_as_float(q[k][i] & 0xFFFF0000u) * 0x1p-4f);
        }
      }
    }

    f32x4d acc[F::NV] = {};
    float off[NG] = {};  // sums of weight times the value of the codes' middle
    float m = LOWEST, l = 0.0f;

    for (int u = ch.b0; u < ch.b1; ++u) {  // the wavefront's steps
      // scores of positions 4 grp + i of tile t
      float x[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x4d sum = {};
        if constexpr (CODES) {
          sum = mfma16(u32x4d{kst[t], kst[t], kst[t], kst[t]}, qs, sum);  // the three terms at once
          const u32x2d st = {kst[t], kst[t]};
#pragma unroll
          for (int e = 0; e < NG; ++e) {
            f32x4d a = {};
#pragma unroll
            for (int k = e * F::NC / NG; k < (e + 1) * F::NC / NG; ++k)
              a = mfma16(key_step<FMT, D>(kw[t], k), q[k], a);
            const f32x4d sc = mfma16(st, u32x2d{pick[e], 0u}, f32x4d{});
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(sc[i], a[i], sum[i]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < F::NC; ++k) sum = mfma16(key_step<FMT, D>(kw[t], k), q[k], sum);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * t + i] = sum[i];
      }
      load_keys();
      const bool tail = nv[0] + nv[1] < 32;
      if (tail) {  // positions that take no part: no weight, and nothing of theirs in the products
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool in = 4 * grp + j % 4 < nv[j / 4];
          x[j] = in ? x[j] : -__builtin_inff();
          if constexpr (!CODES) {
#pragma unroll
            for (int i = 0; i < F::VW; ++i) vw[j][i] = in ? vw[j][i] : 0u;
          }
        }
        if constexpr (CODES) {
#pragma unroll
          for (int t = 0; t < 2; ++t) vst[t] = col < nv[t] ? vst[t] : 0u;
        }
      }
      // running maximum: the reference moves only when a score exceeds it by SLACK
      float mx = x[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, x[j]);
      mx = max4(mx) * cl;
      if (__any(mx > m + SLACK)) {
        const float m1 = fmaxf(m, mx);
        const float f = __builtin_amdgcn_exp2f(m - m1);
        m = m1;
        l *= f;
#pragma unroll
        for (int k = 0; k < F::NV; ++k) acc[k] *= f;
        if constexpr (CODES) {
#pragma unroll
          for (int e = 0; e < NG; ++e) off[e] *= f;
        }
      }
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], cl, -m));
      if (tail) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 4 * grp + j % 4 < nv[j / 4] ? w[j] : 0.0f;
      }
      l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
#pragma unroll
      for (int e = 0; e < NG; ++e) {
        float z[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if constexpr (CODES) {
            const u32x2d st = {vst[t], 0u};
            const f32x4d sc = mfma16(st, u32x2d{pick[e], 0u}, f32x4d{});
            const f32x4d md = mfma16(st, u32x2d{mids[e], 0u}, f32x4d{});
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              z[4 * t + i] = w[4 * t + i] * sc[i];
              off[e] = __builtin_fmaf(w[4 * t + i], md[i], off[e]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * t + i] = w[4 * t + i] * BF16_DOWN;
          }
        }
        u32x4d hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          auto less = [](float v, uint32_t bits, float f) {
            return __builtin_fmaf(v, f, -__uint_as_float(__float_as_uint(v) & bits));
          };
          if constexpr (WIDE) {
            hi[i] = pair(z[2 * i], z[2 * i + 1]);
            lo[i] = pair(less(z[2 * i], 0xFFFF0000u, MORE), less(z[2 * i + 1], 0xFFFF0000u, MORE));
          } else {
            hi[i] = pair(less(z[2 * i], cut, grown), less(z[2 * i + 1], cut, grown));
          }
        }
#pragma unroll
        for (int k = e * F::NV / NG; k < (e + 1) * F::NV / NG; ++k) {
          if constexpr (CODES) {
            const uint32_t bits = FMT == KV_U8 || sixteenfold(k) ? 0x80808080u : 0x80088008u;  // minus the middle, as the codes
            const u32x4d mid = {bits, bits, bits, bits};
            acc[k] = mfma16(mid, hi, acc[k]);
            if constexpr (WIDE) acc[k] = mfma16(mid, lo, acc[k]);
          }
          u32x4d a;
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = value_pair<FMT, D>(vw[2 * i], vw[2 * i + 1], k);
          acc[k] = mfma16(a, hi, acc[k]);
          if constexpr (WIDE) acc[k] = mfma16(a, lo, acc[k]);
        }
      }
      nv[0] = next.nv[0];
      nv[1] = next.nv[1];
      load_values();
    }

    // join the wavefronts: row of column `col` in the order tile, row of the tile
    l = sum4(l);
#pragma unroll
    for (int e = 0; e < NG; ++e) {
      if constexpr (CODES) off[e] = rest ? 0.0f : sum4(off[e]);
#pragma unroll
      for (int k = e * F::NV / NG; k < (e + 1) * F::NV / NG; ++k)
        *reinterpret_cast<f32x4d*>(&so[wave][col][16 * k + 4 * grp]) = CODES ? acc[k] * (sixteenfold(k) ? VBACK / 16 : VBACK) + off[e] : acc[k];
    }
    if (grp == 0) {
      sm[wave][col] = m;
      ss[wave][col] = l;
    }
    more = next_chunk(p, share, ch);
    if (more) load_queries();
    __syncthreads();
    // two neighbouring channels of one head a thread
    for (int o = threadIdx.x; o < HEADS * D / 2; o += 256) {
      const int h = o / (D / 2), cn = o % (D / 2) * 2;
      const int hh = rt * HEADS + h;
      if (hh >= grp_heads) break;
      const int i0 = CODES ? cn : cn % F::NV * 16 + cn / F::NV;
      const int i1 = CODES ? cn + 1 : i0 + 16;
      float top = sm[0][h];
#pragma unroll
      for (int v = 1; v < WAVES; ++v) top = fmaxf(top, sm[v][h]);
      float t = 0.0f, a0 = 0.0f, a1 = 0.0f;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) {
        const float f = __builtin_amdgcn_exp2f(sm[v][h] - top);
        float x0 = so[v][h][i0], x1 = so[v][h][i1];
        if constexpr (!WIDE) {
          x0 += so[v][h + 8][i0];
          x1 += so[v][h + 8][i1];
        }
        t += f * ss[v][h];
        a0 += f * x0;
        a1 += f * x1;
      }
      const int64_t head = int64_t(g) * grp_heads + hh;
      if (opens && closes) {
        const float r = (CODES ? 1.0f : BF16_BACK) / t;
        // no weight at all: 0, where the values may have made the sums NaN
        *reinterpret_cast<uint32_t*>(p.O + s * p.ld_o + head * D + cn) = t == 0.0f ? 0u : pack_bf16x2(a0 * r, a1 * r);
        if (cn == 0 && p.lse) p.lse[s * p.H + head] = t == 0.0f ? -__builtin_inff() : top + __builtin_amdgcn_logf(t);
      } else {
        float* part = chunk(p, want, at, opens, head, D);
        *reinterpret_cast<float2*>(part + 4 + cn) = make_float2(a0, a1);
        if (cn == 0) *reinterpret_cast<float2*>(part) = make_float2(top, t);
      }
    }
    __syncthreads();  // the next chunk writes LDS anew
  }
}

// Joins the chunks of a sequence's head: D / 4 lanes a chunk, PAR chunks at a
// time, four of each in flight.
template <int D>
__global__ __launch_bounds__(512) void attn_join_kernel(AttnDecodeLaunch p, int want) {
  constexpr int LANES = D / 4, PAR = 512 / LANES;
  const int64_t at = workgroup() / p.H;
  const int h = int(workgroup() % p.H);
  if (at >= notes_of(p.c, want)) return;
  const Note note = notes(p)[at];
  if (note.last < 0) return;
  const int s = note.s;
  // share i begins at floor(i total / parts): the last one that begins at note.last or before, counted from the first
  const int n = int(((int64_t(note.last) + 1) * parts_of(note.total, want) - 1) / note.total) - note.share + 1;
  const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
  float m = LOWEST, t = 0.0f;
  f32x4d a = {};
  for (int k = row; k < n; k += 4 * PAR) {
    float2 ml[4];
    f32x4d o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = std::min(k + i * PAR, n - 1);
      const float* part = chunk(p, want, note.share + j, j == 0, h, D);
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
  __shared__ f32x4d so[PAR][LANES];
  __shared__ float sm[PAR], st[PAR];
  so[row][lane] = a;
  if (lane == 0) {
    sm[row] = m;
    st[row] = t;
  }
  __syncthreads();
  if (row) return;
  const int rows = std::min(PAR, n);
  float top = sm[0];
  for (int k = 1; k < rows; ++k) top = fmaxf(top, sm[k]);
  t = 0.0f;
  a = f32x4d{};
  for (int k = 0; k < rows; ++k) {
    const float f = __builtin_amdgcn_exp2f(sm[k] - top);
    t += f * st[k];
    a += f * so[k][lane];
  }
  const float r = (p.c.format == KV_BF16 ? BF16_BACK : 1.0f) / t;
  *reinterpret_cast<uint2*>(p.O + s * p.ld_o + int64_t(h) * D + 4 * lane) =
      t == 0.0f ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(a[0] * r, a[1] * r), pack_bf16x2(a[2] * r, a[3] * r));
  if (lane == 0 && p.lse) p.lse[int64_t(s) * p.H + h] = t == 0.0f ? -__builtin_inff() : top + __builtin_amdgcn_logf(t);
}

// Query heads a workgroup takes, and workgroups a key/value head's heads take.
// More than 8 in tiles of 8, each reading the cache, took 406 us for 64 sequences
// of up to 16384 positions, 128 heads on 8 (with 16 a workgroup 365); 72 heads
// 399 against 355; 48 sequences at 8 bits, 128 heads, 111 against 92.
int row_heads(int H, int H_kv) { return H / H_kv > 8 ? 16 : 8; }
int row_tiles(int H, int H_kv) {
  const int r = row_heads(H, H_kv);
  return (H / H_kv + r - 1) / r;
}

// Shares of each key/value head's row tile for `per` workgroups a CU.
int shares(int64_t n_seq, int H, int H_kv, int64_t max_pages, int page_len, int per) {
  const int64_t most = n_seq * ((max_pages * page_len + BLOCK - 1) / BLOCK + 1) / MIN_COST;
  return int(std::max<int64_t>(1, std::min<int64_t>(most, per * CUS / (int64_t(H_kv) * row_tiles(H, H_kv)))));
}
// Whether a sequence can lie in several shares: not where there is one, nor
// where none is longer than a block.
bool splits(int want, int64_t max_pages, int page_len) { return want > 1 && max_pages * page_len > BLOCK; }

template <int FMT, int D, int NG>
hipError_t launch_form(AttnDecodeLaunch p, hipStream_t st) {
  const int rt = row_tiles(p.H, p.c.H_kv);
  const int want = shares(p.c.n_seq, p.H, p.c.H_kv, p.c.max_pages, p.c.page_len, kResident<FMT, D, NG>);
  if (!splits(want, p.c.max_pages, p.c.page_len)) p.ws = nullptr;
  const int64_t units = (int64_t(want) * p.c.H_kv + 7) / 8 * 8;
  const dim3 grid{unsigned(units * rt)};
  if (p.H / p.c.H_kv > 8)
    attn_decode_kernel<FMT, D, NG, true><<<grid, 256, 0, st>>>(p, want, rt);
  else
    attn_decode_kernel<FMT, D, NG, false><<<grid, 256, 0, st>>>(p, want, rt);
  if (hipError_t e = hipGetLastError()) return e;
  if (!p.ws) return hipSuccess;
  attn_join_kernel<D><<<grid_of(notes_of(p.c, want) * p.H), 512, 0, st>>>(p, want);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const AttnDecodeLaunch& p, hipStream_t st) {
  const bool one = p.c.group == D;
  if (p.c.format == KV_BF16) return launch_form<KV_BF16, D, 1>(p, st);
  if (p.c.format == KV_U8) return one ? launch_form<KV_U8, D, 1>(p, st) : launch_form<KV_U8, D, D / 32>(p, st);
  return one ? launch_form<KV_U4, D, 1>(p, st) : launch_form<KV_U4, D, D / 32>(p, st);
}

}  // namespace

size_t attn_decode_ws(int64_t n_seq, int H, int H_kv, int d, int64_t max_pages, int page_len) {
  const int64_t want = shares(n_seq, H, H_kv, max_pages, page_len, 4);  // the most of any form
  if (!splits(int(want), max_pages, page_len)) return 0;
  return size_t(std::min(n_seq, want)) * 4 + 2 * size_t(want) * size_t(H) * size_t(d + 4);
}

hipError_t launch_attn_decode(const AttnDecodeLaunch& p, hipStream_t st) {
  return p.c.d == 128 ? launch_d<128>(p, st) : launch_d<64>(p, st);
}

}  // namespace uq
