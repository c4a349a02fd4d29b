// The paged key/value cache: new rows written (rotated, quantized) and ranges
// of positions read back.  Layout, quantiser and errors in uniquan.h.
//
// Both are bound by memory: every kernel moves 16 bytes a lane where the
// layout lets it and keeps several rows in flight.  Measured: 8192 rows of 32 + 8
// + 8 heads into an 8-bit cache 185 MB in 36.7 us, 5.0 TB/s; 100002 positions of
// 8 heads from 4 bits to fp32 947 MB (819 of them written) in 230 us, 4.1 TB/s; one row of
// 32 heads 2.6 us, a launch and the loads of its position and page.
//
// Append.  A workgroup takes a row (few rows: a tile of heads of a row).
// Heads that are stored in channel order (queries, keys, values of a bf16
// cache) take D / 16 lanes each, a lane the channels 8 l .. 8 l + 7 and their
// rotary partners D / 2 further on, whose eight (cos, sin) pairs it keeps for
// all its heads; a group of 32 channels is one half of four lanes.  Values
// that become codes take 16 lanes, a lane the channels l + 16 c that lie side
// by side in the row.
//
// Read.  A wavefront takes 16 positions of one head of one sequence, which lie
// on two pages at most, a lane 16 bytes of the output of several.  Its codes of a key are one word (two);
// those of a value lie D / 16 places apart, so a row's lanes exchange them
// through LDS (as byte loads from the cache they took 1.2 to 1.8 times as
// long).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "uq_device.h"
#include "uq_kv.h"
#include "uq_launch.h"

namespace uq {

namespace {

__device__ __forceinline__ float load1(const void* p, int64_t i, bool f32) {
  return f32 ? static_cast<const float*>(p)[i] : bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
}

// 16 bytes that are not read again soon, past the caches (a wavefront writes
// whole lines): 100002 positions of 8 heads to bf16 145 instead of 190 us.
__device__ __forceinline__ void stream16(void* at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  typedef uint32_t u32x4s __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4s{a, b, c, d}, static_cast<u32x4s*>(at));
}

// Minimum, maximum and whether all values are finite.
struct Span {
  float lo, hi;
  bool fine;
};
__device__ __forceinline__ Span join(const Span& a, const Span& b) {
  return Span{fminf(a.lo, b.lo), fmaxf(a.hi, b.hi), a.fine && b.fine};
}
template <int N>
__device__ __forceinline__ Span span_of(const float (&x)[N]) {
  Span s{x[0], x[0], x[0] - x[0] == 0.0f};
#pragma unroll
  for (int i = 1; i < N; ++i) s = join(s, Span{x[i], x[i], x[i] - x[i] == 0.0f});
  return s;
}
// Over LANES neighbouring lanes.
template <int LANES>
__device__ __forceinline__ Span across(Span s) {
#pragma unroll
  for (int m = 1; m < LANES; m <<= 1)
    s = join(s, Span{__shfl_xor(s.lo, m), __shfl_xor(s.hi, m), bool(__shfl_xor(int(s.fine), m))});
  return s;
}

struct Quant {
  float lo, scale, inv;
};

// The stored scale and offset of a group (uniquan.h, "Quantiser").
__device__ __forceinline__ Quant quant_of(const Span& s, float top) {
  Quant q;
  q.lo = bf16_down(s.lo);
  const float spread = s.hi - q.lo;
  if (!s.fine || !(fabsf(spread) <= 3.402823466e38f)) {
    q.lo = q.scale = __uint_as_float(0x7FC00000u);
    q.inv = 0.0f;
    return q;
  }
  q.scale = bf16_up(fmaxf(spread, 0.0f) * (1.0f / top));
  if (q.scale < 1.17549435e-38f) q.scale = 0.0f;
  q.inv = q.scale > 0.0f ? 1.0f / q.scale : 0.0f;
  return q;
}

__device__ __forceinline__ uint32_t code_of(float x, const Quant& q, float top) {
  const float c = rintf((x - q.lo) * q.inv);
  return c == c ? uint32_t(fminf(fmaxf(c, 0.0f), top)) : 0u;
}

// Where a row goes: its sequence, position and page (-1: none).
struct Row {
  int64_t seq;
  int pos, page;
};
// False: padding.
__device__ __forceinline__ bool row_of(const KvAppendLaunch& p, int64_t t, Row& r) {
  const KvCache& c = p.c;
  r.pos = p.pos[t];
  r.seq = p.seq ? p.seq[t] : t;
  if (r.pos < 0 || r.pos >= c.max_pages << c.log_page || (p.cs && r.pos >= p.n_cs) || r.seq < 0 || r.seq >= c.n_seq)
    return false;
  r.page = kv_page(c, r.seq, r.pos);
  return true;
}

// Codes of a run of eight channels of a key, where they lie in the row (in
// bytes): run r at (r % 4)(D / 4) + 8 (r / 4) codes.
template <int D, int FMT>
__device__ __forceinline__ void store_run(uint8_t* row, int r, const float (&x)[8], const Quant& q) {
  const int at = r % 4 * (D / 4) + 8 * (r / 4);
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = code_of(x[i], q, FMT == KV_U8 ? 255.0f : 15.0f);
  if constexpr (FMT == KV_U8) {
    *reinterpret_cast<uint2*>(row + at) =
        make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
  } else {
    *reinterpret_cast<uint32_t*>(row + at / 2) = c[0] | c[2] << 4 | c[4] << 8 | c[6] << 12 | c[1] << 16 | c[3] << 20 |
                                                 c[5] << 24 | c[7] << 28;
  }
}

template <int D, int FMT, bool F32>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendLaunch p) {
  constexpr int LANES = D / 16, SLOTS = 256 / LANES;  // of a head in channel order, heads of a tile
  constexpr int DT = F32 ? DType::F32 : DType::BF16;
  constexpr bool CODES = FMT != KV_BF16;
  constexpr float top = FMT == KV_U8 ? 255.0f : 15.0f;
  constexpr int ROW = FMT == KV_BF16 ? 2 * D : FMT == KV_U8 ? D : D / 2;
  const KvCache& c = p.c;
  const int64_t t = workgroup();
  Row r;
  if (t >= p.T || !row_of(p, t, r)) return;
  const int place = r.pos & (c.page_len - 1);
  const int64_t ph0 = int64_t(r.page) * c.H_kv;
  const int n_q = p.q ? p.H : 0;
  const int plain = n_q + c.H_kv * (CODES ? 1 : 2);  // heads in channel order
  const int tiles = (plain + SLOTS - 1) / SLOTS, vtiles = CODES ? (c.H_kv + 15) / 16 : 0;
  const int lane = threadIdx.x % LANES;
  float co[8], si[8];
  if (p.cs && int(blockIdx.z) < tiles) {
    const float4* cs = reinterpret_cast<const float4*>(p.cs + int64_t(r.pos) * D + 16 * lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 a = cs[i];
      co[2 * i] = a.x;
      si[2 * i] = a.y;
      co[2 * i + 1] = a.z;
      si[2 * i + 1] = a.w;
    }
  }
  for (int tile = blockIdx.z; tile < tiles; tile += gridDim.z) {
    int h = tile * SLOTS + threadIdx.x / LANES;
    if (h >= plain) break;
    const bool is_q = h < n_q, is_k = !is_q && h < n_q + c.H_kv;
    if (!is_q) h -= is_k ? n_q : n_q + c.H_kv;
    if (!is_q && r.page < 0) break;  // queries come first
    const void* src = is_q ? p.q : is_k ? p.k : p.v;
    const int64_t off = t * (is_q ? p.ld_q : is_k ? p.ld_k : p.ld_v) + int64_t(h) * D + 8 * lane;
    float a[8], b[8];
    load8<DT>(src, off, a);
    load8<DT>(src, off + D / 2, b);
    if (p.cs && (is_q || is_k)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x1 = a[i], x2 = b[i];
        a[i] = x1 * co[i] - x2 * si[i];
        b[i] = x2 * co[i] + x1 * si[i];
      }
    }
    const int64_t ph = ph0 + h;
    if (is_q || !CODES) {
      uint16_t* o = is_q ? p.q_out + (t * p.H + h) * D
                         : static_cast<uint16_t*>(is_k ? c.k : c.v) + (ph * c.page_len + place) * D;
      stream16(o + 8 * lane, pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(a[4], a[5]),
               pack_bf16x2(a[6], a[7]));
      stream16(o + 8 * lane + D / 2, pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3]), pack_bf16x2(b[4], b[5]),
               pack_bf16x2(b[6], b[7]));
      continue;
    }
    // a key as codes
    uint8_t* row = static_cast<uint8_t*>(c.k) + (ph * c.page_len + place) * ROW;
    uint32_t* stat = reinterpret_cast<uint32_t*>(c.k_stat) + ph * (D / c.group) * c.page_len + place;
    Span sa = span_of(a), sb = span_of(b);
    if (c.group == 32) {
      const Quant qa = quant_of(across<4>(sa), top), qb = quant_of(across<4>(sb), top);
      store_run<D, FMT>(row, lane, a, qa);
      store_run<D, FMT>(row, lane + D / 16, b, qb);
      if (lane % 4 == 0) {
        stat[lane / 4 * c.page_len] = pack_bf16x2(qa.scale, qa.lo);
        stat[(lane / 4 + D / 64) * c.page_len] = pack_bf16x2(qb.scale, qb.lo);
      }
    } else {
      const Quant q = quant_of(across<LANES>(join(sa, sb)), top);
      store_run<D, FMT>(row, lane, a, q);
      store_run<D, FMT>(row, lane + D / 16, b, q);
      if (lane == 0) stat[0] = pack_bf16x2(q.scale, q.lo);
    }
  }
  if constexpr (CODES) {
    constexpr int N = D / 16;
    if (r.page < 0) return;
    const int l = threadIdx.x & 15;
    for (int tile = int(blockIdx.z) < tiles ? (gridDim.z == 1 ? 0 : vtiles) : int(blockIdx.z) - tiles; tile < vtiles;
         tile += gridDim.z) {
      const int h = tile * 16 + threadIdx.x / 16;
      if (h >= c.H_kv) break;
      const int64_t off = t * p.ld_v + int64_t(h) * D + l;
      float x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = load1(p.v, off + 16 * i, F32);
      const int64_t ph = ph0 + h;
      uint32_t* stat = reinterpret_cast<uint32_t*>(c.v_stat) + ph * (D / c.group) * c.page_len + place;
      uint32_t code[N];
      if (c.group == 32) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const float two[2] = {x[i], x[i + 1]};
          const Quant q = quant_of(across<16>(span_of(two)), top);
          code[i] = code_of(x[i], q, top);
          code[i + 1] = code_of(x[i + 1], q, top);
          if (l == 0) stat[i / 2 * c.page_len] = pack_bf16x2(q.scale, q.lo);
        }
      } else {
        const Quant q = quant_of(across<16>(span_of(x)), top);
#pragma unroll
        for (int i = 0; i < N; ++i) code[i] = code_of(x[i], q, top);
        if (l == 0) stat[0] = pack_bf16x2(q.scale, q.lo);
      }
      uint32_t* row =
          reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(c.v) + (ph * c.page_len + place) * ROW + l * (ROW / 16));
      constexpr int BITS = FMT == KV_U8 ? 8 : 4, PER = 32 / BITS;
      if constexpr (N >= PER) {
#pragma unroll
        for (int w = 0; w < N / PER; ++w) {
          uint32_t v = 0;
#pragma unroll
          for (int i = 0; i < PER; ++i) v |= code[w * PER + i] << (BITS * i);
          row[w] = v;
        }
      } else {
        *reinterpret_cast<uint16_t*>(row) = uint16_t(code[0] | code[1] << 4 | code[2] << 8 | code[3] << 12);
      }
    }
  }
}

constexpr int WAVE_ROWS = 16;  // positions of a wavefront

// N channels from ch on (N divides ch) of a cache row: as they are loaded, which
// for a value's codes is the lane's share of the row.
template <int D, int FMT, bool KEY, int N>
struct Piece {
  static constexpr int ROW = FMT == KV_BF16 ? 2 * D : FMT == KV_U8 ? D : D / 2;
  static constexpr int BYTES = N * ROW / D;
  static constexpr int WORDS = BYTES < 4 ? 1 : BYTES / 4;
  uint32_t w[WORDS], st;

  // at, stat: of the head in its page; lane_stat: of the channels' group there.
  __device__ __forceinline__ void load(const uint8_t* at, const uint32_t* stat, uint32_t place, uint32_t lane_stat,
                                       int ch) {
    at += place * ROW;
    const int run = (ch / 8 % 4 * (D / 4) + 8 * (ch / 32)) * ROW / D;  // of eight channels of a key's codes
    if constexpr (KEY && FMT == KV_U4) {
      w[0] = *reinterpret_cast<const uint32_t*>(at + run) >> (ch % 8 ? 8 : 0);
    } else {
      at += KEY && FMT == KV_U8 ? run + ch % 8 : ch / N * BYTES;
      if constexpr (BYTES == 16) {
        const uint4 v = *reinterpret_cast<const uint4*>(at);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      } else if constexpr (BYTES == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(at);
        w[0] = v.x; w[1] = v.y;
      } else if constexpr (BYTES == 4) {
        w[0] = *reinterpret_cast<const uint32_t*>(at);
      } else {
        w[0] = *reinterpret_cast<const uint16_t*>(at);
      }
    }
    st = FMT == KV_BF16 ? 0u : stat[lane_stat + place];
  }

  // The lane's share of a value's codes to its place in LDS.
  __device__ __forceinline__ void put(uint8_t* row, int ch) const {
    if constexpr (BYTES < 4) {
      *reinterpret_cast<uint16_t*>(row + ch / N * BYTES) = uint16_t(w[0]);
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) *reinterpret_cast<uint32_t*>(row + ch / N * BYTES + 4 * i) = w[i];
    }
  }

  // Channel ch + i; row: a value's codes in LDS.
  __device__ __forceinline__ float value(int i, const uint8_t* row, int ch) const {
    if constexpr (FMT == KV_BF16) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    uint32_t c;
    if constexpr (KEY) {
      c = FMT == KV_U8 ? w[i / 4 % WORDS] >> (8 * (i & 3)) : w[0] >> (4 * (i / 2) + 16 * (i & 1));
    } else {
      const int p = (ch % 16 + i) * (D / 16) + ch / 16;
      c = FMT == KV_U8 ? row[p] : uint32_t(row[p / 2]) >> (4 * (ch / 16 & 1));
    }
    return __uint_as_float(st & 0xFFFF0000u) + __uint_as_float(st << 16) * float(c & (FMT == KV_U8 ? 255u : 15u));
  }
};

template <int D, int FMT, bool F32, bool KEY>
__device__ __forceinline__ void read_rows(const KvReadLaunch& p, void* out, int64_t run, int64_t s, int h, int64_t i0) {
  constexpr int N = F32 ? 4 : 8;  // 16 bytes
  using X = Piece<D, FMT, KEY, N>;
  constexpr int LANES = D / N, PAR = 64 / LANES, ITER = WAVE_ROWS / PAR;
  constexpr bool EXCHANGE = !KEY && FMT != KV_BF16;
  constexpr int LD = X::ROW + (FMT == KV_U8 ? 8 : 4);  // the rows of a wavefront's read on other banks
  __shared__ __attribute__((aligned(16))) uint8_t rows[EXCHANGE ? 4 * WAVE_ROWS * LD : 16];
  const KvCache& c = p.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int ch = lane % LANES * N, row = lane / LANES;
  const int64_t first = (p.start ? p.start[s] : 0) + i0;  // the wavefront's first position
  const int64_t cap = c.max_pages << c.log_page;
  const int64_t end = p.lens[s] < cap ? int64_t(p.lens[s]) : cap;
  // rows [r0, r1) exist, those below cut on the first page, the others on the second
  const int r0 = int(first < 0 ? (first < -WAVE_ROWS ? WAVE_ROWS : -first) : 0);
  const int r1 = int(end - first < 0 ? 0 : end - first < WAVE_ROWS ? end - first : WAVE_ROWS);
  const int64_t from = first < 0 ? 0 : first;
  const int place = int(from & (c.page_len - 1)) - r0, cut = c.page_len - place;
  int page[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t pos = (from >> c.log_page << c.log_page) + k * c.page_len;
    page[k] = r0 < r1 && pos < end ? kv_page(c, s, int(pos)) : -1;
  }
  const uint32_t rows_of_page = uint32_t(c.H_kv) * uint32_t(c.page_len);
  const uint32_t stats = FMT == KV_BF16 ? 0u : uint32_t(D / c.group);
  const uint32_t lane_stat = FMT == KV_BF16 ? 0u : uint32_t(ch / c.group) * c.page_len;
  const uint8_t* at[2];
  const uint32_t* stat[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint64_t pg = page[k] < 0 ? 0u : uint32_t(page[k]);
    at[k] = static_cast<const uint8_t*>(KEY ? c.k : c.v) + pg * (rows_of_page * X::ROW) + uint32_t(h) * c.page_len * X::ROW;
    stat[k] = reinterpret_cast<const uint32_t*>(KEY ? c.k_stat : c.v_stat) + pg * (rows_of_page * stats) +
              uint32_t(h) * stats * c.page_len;
  }
  X x[ITER];
  bool is[ITER];
#pragma unroll
  for (int j = 0; j < ITER; ++j) {
    const int r = j * PAR + row;
    const bool second = r >= cut;
    is[j] = r >= r0 && r < r1 && (second ? page[1] : page[0]) >= 0;
    if (is[j])
      x[j].load(second ? at[1] : at[0], second ? stat[1] : stat[0], uint32_t(second ? r - cut : place + r), lane_stat, ch);
  }
  uint8_t* mine = rows + (EXCHANGE ? (wave * WAVE_ROWS + row) * LD : 0);
  if constexpr (EXCHANGE) {  // within a row's lanes
#pragma unroll
    for (int j = 0; j < ITER; ++j) x[j].put(mine + j * PAR * LD, ch);
    wave_lds_sync();
  }
  const int64_t o = (run + i0 + row) * D + ch;
  const int left = int(p.L - i0 < WAVE_ROWS ? p.L - i0 : WAVE_ROWS);
#pragma unroll
  for (int j = 0; j < ITER; ++j) {
    if (j * PAR + row >= left) break;
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = is[j] ? x[j].value(e, mine + j * PAR * LD, ch) : 0.0f;
    if constexpr (F32)
      stream16(static_cast<float*>(out) + o + j * PAR * D, __float_as_uint(v[0]), __float_as_uint(v[1]),
               __float_as_uint(v[2]), __float_as_uint(v[3]));
    else
      stream16(static_cast<uint16_t*>(out) + o + j * PAR * D, pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
               pack_bf16x2(v[4 % N], v[5 % N]), pack_bf16x2(v[6 % N], v[7 % N]));
  }
}

template <int D, int FMT, bool F32>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadLaunch p) {
  // wavefront's (side, head, sequence, 16 positions), the keys first; fewer than 2^30 of them
  const uint32_t per = uint32_t((p.L + WAVE_ROWS - 1) / WAVE_ROWS), n_seq = uint32_t(p.c.n_seq);
  const uint32_t one = uint32_t(p.c.H_kv) * n_seq;
  const uint32_t unit = uint32_t(workgroup()) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t hs = unit / per;
  const int64_t i0 = int64_t(unit % per) * WAVE_ROWS;
  const bool key = p.K && hs < one;
  if (p.K && !key) hs -= one;
  if (hs >= one || (!key && !p.V)) return;
  const int h = int(hs / n_seq);
  const int64_t s = hs % n_seq;
  if (key)
    read_rows<D, FMT, F32, true>(p, p.K, hs * p.L, s, h, i0);
  else
    read_rows<D, FMT, F32, false>(p, p.V, hs * p.L, s, h, i0);
}

}  // namespace

namespace {

template <int D, int FMT, bool F32>
void append_form(const KvAppendLaunch& p, hipStream_t st) {
  constexpr int SLOTS = 256 * 16 / D;
  const int plain = (p.q ? p.H : 0) + p.c.H_kv * (FMT == KV_BF16 ? 2 : 1);
  const int tiles = (plain + SLOTS - 1) / SLOTS + (FMT == KV_BF16 ? 0 : (p.c.H_kv + 15) / 16);
  // Few rows: a workgroup for every tile of heads (32 + 8 heads at 8 bits, one row 3.0 us against 4.3 with
  // a workgroup a row, 1024 rows 9.2 against 9.7); many: a row's tiles share its angles (2048 rows 14.8
  // against 15.9, 4096 29.6 against 32.4).
  dim3 grid = grid_of(p.T);
  grid.z = p.T < 1536 ? unsigned(tiles) : 1u;
  kv_append_kernel<D, FMT, F32><<<grid, 256, 0, st>>>(p);
}
template <int D>
void append_d(const KvAppendLaunch& p, hipStream_t st) {
  const bool f32 = p.in_dtype == F32;
  switch (p.c.format) {
    case KV_BF16: return f32 ? append_form<D, KV_BF16, true>(p, st) : append_form<D, KV_BF16, false>(p, st);
    case KV_U8: return f32 ? append_form<D, KV_U8, true>(p, st) : append_form<D, KV_U8, false>(p, st);
    default: return f32 ? append_form<D, KV_U4, true>(p, st) : append_form<D, KV_U4, false>(p, st);
  }
}

template <int D, int FMT>
void read_form(const KvReadLaunch& p, hipStream_t st) {
  const int sides = (p.K ? 1 : 0) + (p.V ? 1 : 0);
  const int64_t units = sides * p.c.H_kv * p.c.n_seq * ((p.L + WAVE_ROWS - 1) / WAVE_ROWS);
  const dim3 grid = grid_of((units + 3) / 4);
  if (p.out_dtype == F32)
    kv_read_kernel<D, FMT, true><<<grid, 256, 0, st>>>(p);
  else
    kv_read_kernel<D, FMT, false><<<grid, 256, 0, st>>>(p);
}
template <int D>
void read_d(const KvReadLaunch& p, hipStream_t st) {
  switch (p.c.format) {
    case KV_BF16: return read_form<D, KV_BF16>(p, st);
    case KV_U8: return read_form<D, KV_U8>(p, st);
    default: return read_form<D, KV_U4>(p, st);
  }
}

}  // namespace

hipError_t launch_kv_append(const KvAppendLaunch& p, hipStream_t st) {
  if (p.c.d == 128)
    append_d<128>(p, st);
  else
    append_d<64>(p, st);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvReadLaunch& p, hipStream_t st) {
  if (p.c.d == 128)
    read_d<128>(p, st);
  else
    read_d<64>(p, st);
  return hipGetLastError();
}

}  // namespace uq
