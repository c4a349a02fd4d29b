// One token per row of logits (uniquan_sample); definition and errors in
// uniquan.h.
//
// Weights.  w = rint(2^sh e^((x - max) / t)), sh = min(51, 62 - ceil(log2 V)):
// integers whose sums are exact and the same in any order, so that every comparison
// of a running sum with a border has one answer however the work is split.  The
// exponential is taken in 64 bits: with one in 32 bits the running sums of some
// ten thousand tokens are off by 1e-7 of their total, and a random number falls that
// near to one of the borders once in some hundred rows.
//
// A workgroup takes a row and reads it once per pass (the first time from memory,
// then from the caches):
//   maximum    of every lane's tokens and of all: also the greedy answer.
//   top-k of up to ENOUGH: the k-th best of the lanes' best tokens is a value that k
//              tokens reach at least, and few more.  They are gathered in LDS, and
//              everything else happens there.
//   min-p      alike, where the lanes' best tokens say that few are left.
//   histogram  (top-p, larger k) counts and sums of weights in BINS equal steps of
//              (max - x) / t: its running sums say in which bin the k-th token lies
//              and in which the nucleus ends.  A nucleus of up to CAP tokens is
//              gathered too; else the bin in which the cut lies, to find it exactly.
//              A bin of more than CAP tokens is cut by further histograms, of equal
//              steps between its smallest and largest value; many tokens of one value
//              by their indices.
//   sums       of the weights kept, a sixteenth of the indices a wavefront, then of
//              the one in whose share u times the total falls, and so on.
// Up to FEW gathered tokens are not sorted: 1024 / n threads a token go through the
// others for its rank and the sums before it (of 1024 tokens that takes 55 us, their
// sorting 4).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "uq_device.h"
#include "uq_kv.h"
#include "uq_launch.h"

namespace uq {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int BINS = 2048;   // two a thread
constexpr int CAP = 1024;    // tokens gathered in LDS
constexpr int FEW = 128;     // of those that are not sorted
constexpr int ENOUGH = 512;  // best tokens of lanes that are asked for

typedef unsigned long long u64;

// x, the same in every lane, in scalar registers.
__device__ __forceinline__ uint32_t uni(uint32_t x) { return uint32_t(__builtin_amdgcn_readfirstlane(int(x))); }
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uni(float x) { return __uint_as_float(uni(__float_as_uint(x))); }
__device__ __forceinline__ u64 uni(u64 x) { return u64(uni(uint32_t(x >> 32))) << 32 | uni(uint32_t(x)); }
__device__ __forceinline__ double uni(double x) { return __longlong_as_double((long long)uni(u64(__double_as_longlong(x)))); }

// Order of the tokens, best first: larger values, then lower indices.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return ~(b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u));
}
__device__ __forceinline__ float value_of(uint32_t key) {
  const uint32_t u = ~key;
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ u64 place_of(float x, int i) { return u64(key_of(x)) << 32 | uint32_t(i); }

__device__ __forceinline__ u64 shfl_xor(u64 x, int d) {
  return u64(__shfl_xor(uint32_t(x >> 32), d)) << 32 | __shfl_xor(uint32_t(x), d);
}
// x of the lane that a DPP control names, 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, uint32_t(x), CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, uint32_t(x >> 32), CTRL, ROWS, 0xF, false);
  return u64(hi) << 32 | lo;
}
// Sum over the lanes up to this one.
__device__ __forceinline__ u64 wave_upto(u64 x) {
  x += moved<0x111, 0xF>(x);  // row_shr:1
  x += moved<0x112, 0xF>(x);
  x += moved<0x114, 0xF>(x);
  x += moved<0x118, 0xF>(x);
  x += moved<0x142, 0xA>(x);  // row_bcast:15
  x += moved<0x143, 0xC>(x);  // row_bcast:31
  return x;
}
__device__ __forceinline__ u64 wave_sum(u64 x) {
  x = wave_upto(x);
  return u64(uint32_t(__builtin_amdgcn_readlane(uint32_t(x >> 32), 63))) << 32 |
         uint32_t(__builtin_amdgcn_readlane(uint32_t(x), 63));
}

struct Lds {
  u64 mass[BINS];
  uint32_t count[BINS];
  u64 list[CAP], weight[FEW];
  u64 wave[WAVES];
  u64 found[4];
  uint32_t n, lo, hi;
  float top[WAVES];
};

// Sum over the workgroup's threads before this one; all: of all of them.
__device__ __forceinline__ u64 block_before(Lds& s, u64 x, u64& all) {
  const int wave = threadIdx.x >> 6;
  const u64 upto = wave_upto(x);
  __syncthreads();  // s.wave is free
  if ((threadIdx.x & 63) == 63) s.wave[wave] = upto;
  __syncthreads();
  u64 before = 0;
  all = 0;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    const u64 y = s.wave[v];
    before += v < wave ? y : 0;
    all += y;
  }
  return before + upto - x;
}

// What a row without a whole chunk loads in place of one.
__device__ const uint4 no_chunk = {};

// A row as aligned chunks of 16 bytes, the first and the last in part.
template <bool F32>
struct Row {
  static constexpr int E = F32 ? 4 : 8;
  static constexpr uint32_t NONE = F32 ? 0xFF800000u : 0xFF80FF80u;  // -infinity
  const char* at;  // of chunk 0
  int shift;       // elements of chunk 0 before the row
  int V, chunks;
  int per;         // chunks of a lane: a wavefront's lie side by side
  int lo, hi;      // the whole chunks (lo > hi: none)

  __device__ Row(const void* x, int64_t off, int V) : V(V) {
    const char* p = static_cast<const char*>(x) + off * (F32 ? 4 : 2);
    const int over = int(reinterpret_cast<uintptr_t>(p) & 15);
    at = p - over;
    shift = over / (F32 ? 4 : 2);
    chunks = (shift + V + E - 1) / E;
    per = (chunks + THREADS - 1) / THREADS;
    lo = shift > 0;
    hi = (shift + V) / E - 1;
  }
  __device__ __forceinline__ int chunk(int wave, int i) const { return (wave * per + i) * 64 + int(threadIdx.x & 63); }
  __device__ __forceinline__ int first(int c) const { return c * E - shift; }
  // Words of chunk c, without a branch: of one in part, or of none, some other's.  (Named global: the compiler
  // does not see it through the choice, and a wait for one of its flat loads is one for all of them.)
  __device__ __forceinline__ uint4 ask(int c) const {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef const __attribute__((address_space(1))) u32x4 Global;
    const uintptr_t p = reinterpret_cast<uintptr_t>(lo <= hi ? static_cast<const void*>(at) : &no_chunk);
    const u32x4 q = reinterpret_cast<Global*>(p)[lo <= hi ? min(max(c, lo), hi) : 0];
    return make_uint4(q.x, q.y, q.z, q.w);
  }
  // The words asked for, or those of a chunk in part; what is outside the row is -infinity.
  __device__ __forceinline__ uint4 get(int c, uint4 q) const {
    if (!__any(c < lo || c > hi)) return q;
    uint4 part = make_uint4(NONE, NONE, NONE, NONE);
    if (__any((c < lo || c > hi) && c < chunks)) {
#pragma unroll 1
      for (int e = 0; e < E; ++e) {  // moved in from behind
        const int i = first(c) + e;
        const bool in = i >= 0 && i < V;
        if constexpr (F32) {
          const uint32_t v = in ? reinterpret_cast<const uint32_t*>(at)[int64_t(c) * E + e] : NONE;
          part = make_uint4(part.y, part.z, part.w, v);
        } else {
          const uint32_t v = in ? reinterpret_cast<const uint16_t*>(at)[int64_t(c) * E + e] : 0xFF80u;
          part = make_uint4(part.x >> 16 | part.y << 16, part.y >> 16 | part.z << 16, part.z >> 16 | part.w << 16,
                            part.w >> 16 | v << 16);
        }
      }
    }
    return c < lo || c > hi ? part : q;
  }
  __device__ __forceinline__ uint4 load(int c) const { return get(c, ask(c)); }
  // Element e of a chunk as it stands.
  static __device__ __forceinline__ float raw(const uint4& c, int e) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    return F32 ? __uint_as_float(w[e]) : __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
};

// f(chunk, its words) for chunk groups [i0, i1) of wavefront `of`; the wavefront stays
// together (chunks behind the end are -infinity).  Four chunks are on their way while
// one is worked on.  The loop is not unrolled: a row is few iterations, and code that
// runs once is bound by its own loads (with eight chunks in registers and their code in
// a row, the maximum of 32000 logits took 18 us in place of 9).
template <bool F32, typename Fn>
__device__ __forceinline__ void over_chunks(const Row<F32>& row, int of, int i0, int i1, Fn f) {
  auto at = [&](int i) { return row.chunk(of, i); };
  uint4 a = row.ask(at(i0)), b = row.ask(at(i0 + 1)), c = row.ask(at(i0 + 2)), d = row.ask(at(i0 + 3));
#pragma unroll 1
  for (int i = i0; i < i1; ++i) {
    const uint4 q = row.get(at(i), a);
    a = b;
    b = c;
    c = d;
    d = row.ask(at(i + 4));
    f(at(i), q);
  }
}
// A logit as it counts: NaN as -infinity, -0 as 0.
__device__ __forceinline__ float clean(float x) { return x == x ? x + 0.0f : -__builtin_inff(); }

// f(four elements as they stand, the first one's index) for their elements; only of
// chunks that have one of `from` or more in some lane.
template <bool F32, typename Fn>
__device__ __forceinline__ void over_fours(const Row<F32>& row, int of, int i0, int i1, float from, Fn f) {
  over_chunks(row, of, i0, i1, [&](int c, uint4 q) {
    float m = row.raw(q, 0);
#pragma unroll
    for (int e = 1; e < Row<F32>::E; ++e) m = fmaxf(m, row.raw(q, e));  // (not NaN, if there is another)
    if (!__any(m >= from)) return;
    int i = row.first(c);
#pragma unroll 1
    for (int h = 0; h < Row<F32>::E / 4; ++h, i += 4) {
      const float x[4] = {row.raw(q, 0), row.raw(q, 1), row.raw(q, 2), row.raw(q, 3)};
      f(x, i);
      q = make_uint4(q.z, q.w, q.z, q.w);
    }
  });
}
// f(x, index) for them, one after the other.
template <bool F32, typename Fn>
__device__ __forceinline__ void over_part(const Row<F32>& row, int of, int i0, int i1, float from, Fn f) {
  over_fours(row, of, i0, i1, from, [&](const float (&x)[4], int i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f(x[e], i + e);
  });
}
template <bool F32, typename Fn>
__device__ __forceinline__ void over_row(const Row<F32>& row, float from, Fn f) {
  over_part(row, uni(int(threadIdx.x >> 6)), 0, row.per, from, f);
}

// A token's weight in units of 2^-sh: 2^y, y = n + r with r in [-1/2, 1/2], by the
// polynomial of degree 10 through 2^r at the 11 Chebyshev points (off by 3e-16 of
// it at most); n + sh from the low bits of a sum with 2^52 and into the exponent by an
// integer addition.  20 instructions; with the library's exponential and conversions
// a pass took three times as long.
__constant__ const double kPower[11] = {  // highest first
    7.07258594926922339e-09, 1.02086902999583060e-07, 1.32154425879216893e-06,
    1.52526572602008367e-05, 1.54035304417360499e-04, 1.33335582301649744e-03,
    9.61812910760688825e-03, 5.55041086644477225e-02, 2.40226506959100972e-01,
    6.93147180559949949e-01, 1.00000000000000000e+00};

// a b + c with c in scalar registers, which the compiler copies to vector registers
// first (11 pairs of them, for which others went to memory).
__device__ __forceinline__ double fma_s(double a, double b, double c) {
  double d;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(c));
  return d;
}

struct Weigh {
  float top;       // the row's maximum, 0 where that is +infinity
  bool endless;    // it is: tokens at it count as 0, others as -infinity
  double per_t;    // log2(e) / temperature
  double least;    // of x - max, -1000 / per_t: the weight rounds to 0
  double magic;    // 1.5 2^52 + sh
  double lead;     // the power's first coefficient
  float bins;      // bins per unit of max - x
  float width;     // of a bin

  // A logit as it stands, for a row of +infinity's.
  __device__ __forceinline__ float seen(float x) const {
    return endless ? (x == __builtin_inff() ? 0.0f : -__builtin_inff()) : x;
  }
  // Monotone in x; weights in the last bin are 0.
  __device__ __forceinline__ int bin(float x) const { return int(fminf((top - x) * bins, float(BINS - 1))); }
  // Values of bin b lie in [floor_of(b), ceil_of(b)]: a bin to spare for the roundings.
  __device__ __forceinline__ float floor_of(int b) const { return uni(top - float(b + 2) * width); }
  __device__ __forceinline__ float ceil_of(int b) const { return uni(b < 2 ? top : top - float(b - 1) * width); }
  // The weights of N tokens above BIAS, step by step side by side.
  static constexpr u64 BIAS = u64(0x433) << 52;
  template <int N>
  __device__ __forceinline__ void biased(const float (&x)[N], u64 (&w)[N]) const {
    double t[N], r[N], v[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {  // (-infinity and NaN as the least)
      r[e] = fmax(double(x[e]) - double(top), least);
      t[e] = fma(r[e], per_t, magic);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = fma(r[e], per_t, magic - t[e]);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = fma_s(r[e], lead, kPower[1]);
#pragma unroll
    for (int i = 2; i < 11; ++i) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = fma_s(v[e], r[e], kPower[i]);
    }
    // 2^(n + sh) times it, rounded to an integer in the low bits
#pragma unroll
    for (int e = 0; e < N; ++e) {
      v[e] = __hiloint2double(__double2hiint(v[e]) + (__double2loint(t[e]) << 20), __double2loint(v[e])) + 0x1p52;
      w[e] = u64(__double_as_longlong(v[e]));
    }
  }
  __device__ __forceinline__ u64 operator()(float x) const {
    const float one[1] = {x};
    u64 v[1];
    biased(one, v);
    return v[0] - BIAS;
  }
};

// A cut in the order of the tokens: the first `count` of them, or, where by_mass,
// those before which the weights sum to less than `mass`.
struct Cut {
  bool by_mass;
  uint32_t count;
  u64 mass;
};

// Running sums of the histogram before each thread's bins 2 i and 2 i + 1; of the
// weights where MASS, else 0.
struct Before {
  uint32_t c[2], all_c;
  u64 m[2];
};
template <bool MASS>
__device__ __forceinline__ Before bins_before(Lds& s, u64& all) {
  const int b = 2 * threadIdx.x;
  const uint32_t c0 = s.count[b], c1 = s.count[b + 1];
  u64 counted;
  Before r{};
  all = 0;
  r.c[0] = uint32_t(block_before(s, u64(c0) + c1, counted));
  r.all_c = uint32_t(counted);
  r.c[1] = r.c[0] + c0;
  if constexpr (MASS) {
    const u64 m0 = s.mass[b], m1 = s.mass[b + 1];
    r.m[0] = block_before(s, m0 + m1, all);
    r.m[1] = r.m[0] + m0;
  }
  return r;
}

__device__ __forceinline__ void clear_bins(Lds& s) {
  __syncthreads();
  for (int b = threadIdx.x; b < BINS; b += THREADS) {
    s.mass[b] = 0;
    s.count[b] = 0;
  }
  __syncthreads();
}

// The bin in which the cut lies, the one that its sums reach first; the sums before
// it.  (A cut behind all tokens that are counted lies in the last one's bin.)
__device__ __forceinline__ int bin_of_cut(Lds& s, const Before& r, const Cut& cut, uint32_t& c, u64& m) {
  const uint32_t count = min(cut.count, r.all_c);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int b = 2 * threadIdx.x + i;
    if (cut.by_mass ? r.m[i] < cut.mass && cut.mass <= r.m[i] + s.mass[b] : r.c[i] < count && count <= r.c[i] + s.count[b]) {
      s.found[0] = b;
      s.found[1] = r.c[i];
      s.found[2] = r.m[i];
    }
  }
  __syncthreads();
  c = uni(uint32_t(s.found[1]));
  m = uni(s.found[2]);
  const int b = uni(int(s.found[0]));
  __syncthreads();
  return b;
}

// The wavefront in whose sum `at` (below the total) falls; left: at less the sums before it.
__device__ __forceinline__ int pick(Lds& s, u64 sum, u64 at, u64& left) {
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.wave[threadIdx.x >> 6] = sum;
  __syncthreads();
  int v = 0;
  while (v < WAVES - 1 && s.wave[v] <= at) at -= s.wave[v++];
  left = uni(at);
  return uni(v);
}

// f(x, index) of `from` and larger go to the list as far as it goes; s.n counts them all.
template <bool F32, typename Keep>
__device__ __forceinline__ void gather(Lds& s, const Row<F32>& row, const Weigh& w, float from, Keep keep) {
  __syncthreads();
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  over_row(row, w.endless ? __builtin_inff() : from, [&](float x, int i) {
    x = w.seen(x);
    if (!(x >= from)) return;
    x = clean(x);
    if (!keep(x)) return;
    const uint32_t at = atomicAdd(&s.n, 1u);
    if (at < CAP) s.list[at] = place_of(x, i);
  });
  __syncthreads();
}

// The n numbers x of threads 0 .. n - 1 (n > 64), ~0 elsewhere, in ascending order.
__device__ __forceinline__ u64 sorted(Lds& s, u64 x, uint32_t n) {
  const uint32_t me = threadIdx.x;
#pragma unroll 1
  for (uint32_t k = 2; k < 2 * n; k <<= 1) {
#pragma unroll 1
    for (uint32_t j = k / 2; j > 0; j >>= 1) {
      u64 y;
      if (j < 64) {
        y = shfl_xor(x, int(j));
      } else {
        __syncthreads();
        s.list[me] = x;
        __syncthreads();
        y = s.list[me ^ j];
      }
      const bool low = ((me & j) == 0) == ((me & k) == 0);
      x = (x < y) == low ? x : y;
    }
  }
  return x;
}

// A gathered token: thread `part` of the `parts` neighbouring ones that have it.
struct Token {
  bool is;
  int parts, part;
  u64 place, mine;   // its weight
  uint32_t rank;     // tokens before it in order
  u64 before;        // their weights
};
// Sum over the threads of a token, in all of them.
__device__ __forceinline__ u64 over_parts(u64 x, int parts) {
  for (int d = 1; d < parts; d <<= 1) x += shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ Token rank_list(Lds& s, const Weigh& w, uint32_t n) {
  Token t;
  const uint32_t me = threadIdx.x;
  if (n > FEW) {
    t.parts = 1;
    t.part = 0;
    t.is = me < n;
    t.place = t.is ? s.list[me] : ~u64(0);
    t.place = sorted(s, t.place, n);
    t.mine = t.is ? w(value_of(uint32_t(t.place >> 32))) : 0;
    u64 all;
    t.before = block_before(s, t.mine, all);
    t.rank = me;
    return t;
  }
  t.parts = n <= THREADS / 32 ? 32 : THREADS / FEW;
  t.part = me & (t.parts - 1);
  const uint32_t i = me / t.parts;
  t.is = i < n;
  if (me < n) s.weight[me] = w(value_of(uint32_t(s.list[me] >> 32)));
  __syncthreads();
  t.place = t.is ? s.list[i] : 0;
  t.mine = t.is ? s.weight[i] : 0;
  uint32_t rank = 0;
  u64 before = 0;
  for (uint32_t j = t.part; j < n; j += t.parts) {
    const bool better = s.list[j] < t.place;
    rank += better;
    before += better ? s.weight[j] : 0;
  }
  t.before = over_parts(before, t.parts);
  t.rank = uint32_t(over_parts(rank, t.parts));
  return t;
}

// The cut among the tokens of bin b (n of them): place of the last one before it, and the sum of the weights there.
// (Inlined in any case: called, its registers and the LDS by plain addresses cost bf16 rows 15 of 65 us.)
template <bool F32>
__device__ __forceinline__ u64 cut_bin(Lds& s, const Row<F32>& row, const Weigh& w, int b, uint32_t n, Cut cut, u64& mass) {
  uint32_t lo = 0, hi = ~0u;  // keys still in question
  mass = 0;
  const float from = w.floor_of(b), to = w.ceil_of(b);
  // f(x, its key) for the tokens in question
  auto over_bin = [&](auto f) {
    over_row(row, w.endless ? __builtin_inff() : from, [&](float x, int) {
      x = w.seen(x);
      if (!(x >= from && x <= to)) return;
      x = clean(x);
      const uint32_t k = key_of(x);
      if (w.bin(x) == b && k >= lo && k <= hi) f(x, k);
    });
  };
  while (n > CAP) {
    __syncthreads();
    if (threadIdx.x == 0) {
      s.lo = ~0u;
      s.hi = 0;
    }
    __syncthreads();
    uint32_t a = ~0u, z = 0;
    over_bin([&](float, uint32_t k) {
      a = min(a, k);
      z = max(z, k);
    });
    atomicMin(&s.lo, a);
    atomicMax(&s.hi, z);
    __syncthreads();
    lo = uni(s.lo);
    hi = uni(s.hi);
    if (lo == hi) break;
    clear_bins(s);
    const int drop = std::max(0, 32 - __builtin_clz(hi - lo) - 11);  // (hi - lo) >> drop is below BINS
    over_bin([&](float x, uint32_t k) {
      atomicAdd(&s.count[(k - lo) >> drop], 1u);
      atomicAdd(&s.mass[(k - lo) >> drop], w(x));
    });
    __syncthreads();
    u64 all;
    const Before r = bins_before<true>(s, all);
    uint32_t c;
    u64 m;
    const int v = bin_of_cut(s, r, cut, c, m);
    n = uni(s.count[v]);
    cut.count -= cut.by_mass ? 0 : c;
    cut.mass -= cut.by_mass ? m : 0;
    mass += m;
    hi = lo + uint32_t(((u64(v) + 1) << drop) - 1);
    lo += uint32_t(v) << drop;
  }
  if (n > CAP) {  // one value: the first r of them by index
    const u64 one = w(value_of(lo));
    u64 r = cut.by_mass ? (one ? (cut.mass + one - 1) / one : n) : cut.count;
    r = r < n ? r : n;
    mass += r * one;
    if (r == n) return u64(lo) << 32 | 0x7FFFFFFFu;  // all of them (the bin may hold lower values: behind any index)
    // how many lie in each wavefront's share of the indices, then in each of its chunk groups
    const float only = value_of(lo);
    auto same = [&](float x) { return clean(w.seen(x)) == only; };
    const float any = -__builtin_inff();
    u64 mine = 0;
    over_row(row, any, [&](float x, int) { mine += same(x); });
    const int wave = pick(s, wave_sum(mine), r - 1, r);  // r: what is left, counted from 0
    for (int i = 0; i < row.per && int(threadIdx.x >> 6) == wave; ++i) {
      u64 here = 0;
      over_part(row, wave, i, i + 1, any, [&](float x, int) { here += same(x); });
      const u64 upto = wave_upto(here), end = wave_sum(here);
      if (r >= end) {
        r -= end;
        continue;
      }
      u64 at = upto - here;
      over_part(row, wave, i, i + 1, any, [&](float x, int j) {
        if (same(x) && at++ == r) s.found[3] = place_of(only, j);
      });
      break;
    }
    __syncthreads();
    return s.found[3];
  }
  gather(s, row, w, from, [&](float x) {
    const uint32_t k = key_of(x);
    return x <= to && w.bin(x) == b && k >= lo && k <= hi;
  });
  if (threadIdx.x < 2) s.found[threadIdx.x] = 0;
  const Token t = rank_list(s, w, n);
  if (t.is && t.part == 0 && (cut.by_mass ? t.before < cut.mass : t.rank < cut.count)) {
    atomicMax(&s.found[0], t.place);
    atomicMax(&s.found[1], t.before + t.mine);
  }
  __syncthreads();
  mass += s.found[1];
  return s.found[0];
}

// Counts and sums of weights per bin, and the sums before each thread's bins.
template <bool F32>
__device__ __forceinline__ Before histogram(Lds& s, const Row<F32>& row, const Weigh& w, u64& total) {
  clear_bins(s);
  const float from = w.floor_of(BINS - 2);  // the last bin's tokens, and what is outside the row, have no weight
  over_fours(row, uni(int(threadIdx.x >> 6)), 0, row.per, w.endless ? __builtin_inff() : from, [&](const float (&in)[4], int) {
    float x[4] = {in[0], in[1], in[2], in[3]};
    if (w.endless) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = w.seen(x[e]);
    }
    u64 v[4];
    w.biased(x, v);
    int b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = x[e] >= from ? w.bin(x[e]) : BINS - 1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (b[e] == BINS - 1) continue;
      atomicAdd(&s.count[b[e]], 1u);
      atomicAdd(&s.mass[b[e]], v[e] - Weigh::BIAS);
    }
  });
  __syncthreads();
  return bins_before<true>(s, total);
}

// Sum of the lane's weights of the tokens up to end_x, end_i in order, in a row without +infinity: what is behind
// counts as -infinity, and four chains have no branch (one after the other, with the tests of the general case, 256 x
// 131072 logits took 55 us in place of 37).
template <bool F32>
__device__ __forceinline__ u64 mass_upto(const Row<F32>& row, const Weigh& w, int of, int i0, int i1, float end_x, int end_i) {
  const float past_x = uni(value_of(key_of(end_x) - 1));  // the next larger value
  u64 sum = 0;
  uint32_t n = 0;
  over_fours(row, of, i0, i1, end_x, [&](const float (&x)[4], int i) {
    const float least_x = i <= end_i ? end_x : past_x;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = x[e] >= least_x ? x[e] : -__builtin_inff();
    if (i <= end_i && end_i < i + 3) {
#pragma unroll
      for (int e = 1; e < 4; ++e) y[e] = i + e <= end_i || x[e] > end_x ? y[e] : -__builtin_inff();
    }
    u64 v[4];
    w.biased(y, v);
    sum += (v[0] + v[1]) + (v[2] + v[3]);
    n += 4;
  });
  return sum - n * Weigh::BIAS;
}

// floor(u total) for u in [0, 1); the last unit from 1 on.
__device__ __forceinline__ u64 part_of(float u, u64 total) {
  if (!(u > 0.0f)) return 0;
  if (u >= 1.0f) return total - 1;
  return __umul64hi(u64(double(u) * 0x1p64), total);
}

// Whether sums below it are below p total, p < 1: ceil(p total), and 1 at least, the first token (also where p is
// below 2^-64).
__device__ __forceinline__ u64 border_of(float p, u64 total) {
  if (!(p > 0.0f)) return 1;
  const u64 f = u64(double(p) * 0x1p64), hi = __umul64hi(f, total), lo = f * total;
  return std::max<u64>(hi + (lo != 0), 1);
}

// The answer from the gathered tokens, if they are not too many and hold all that
// stays.  total: the weights' sum over the row where top-k is off; all: they do, by min_p.
template <typename Answer>
__device__ __forceinline__ bool answer_of_list(Lds& s, const Weigh& w, uint32_t k, float top_p, u64 least, u64 total,
                                               bool all, float u, Answer answer) {
  const uint32_t n = uni(s.n);
  if (n > CAP) return false;
  if (threadIdx.x == 0) s.found[0] = 0;
  const Token t = rank_list(s, w, n);
  const bool first = t.is && t.part == 0;
  if (first && (!k || t.rank < k)) atomicMax(&s.found[0], t.before + t.mine);
  __syncthreads();
  const u64 held = s.found[0], border = top_p < 1.0f ? border_of(top_p, k ? held : total) : ~u64(0);
  if (top_p < 1.0f && border > held && !all) return false;
  const bool stays = t.is && (!k || t.rank < k) && t.before < border && t.mine >= least;
  u64 place = t.place, mine = stays ? t.mine : 0, upto = 0, sum = 0;
  if (n > FEW) {  // by index, what does not stay behind
    place = sorted(s, stays ? place << 32 | place >> 32 : ~u64(0), n);
    mine = place == ~u64(0) ? 0 : w(value_of(uint32_t(place)));
    upto = block_before(s, mine, sum);
    place >>= 32;
  } else {
    if (first) s.weight[threadIdx.x / t.parts] = mine;
    __syncthreads();
    for (uint32_t j = t.part; j < n; j += t.parts) {
      const u64 v = s.weight[j];
      sum += v;
      upto += uint32_t(s.list[j]) < uint32_t(place) ? v : 0;
    }
    upto = over_parts(upto, t.parts);
    sum = over_parts(sum, t.parts);
  }
  const u64 target = part_of(u, sum);
  if (t.part == 0 && upto <= target && target < upto + mine) answer(int(uint32_t(place)), float(double(mine) / double(sum)));
  return true;
}

template <bool F32>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleLaunch p) {
  __shared__ Lds s;
  const int64_t t = workgroup();
  if (t >= p.T) return;
  const Row<F32> row(p.x, t * p.ld, p.V);
  const int lane = threadIdx.x & 63, wave = uni(int(threadIdx.x >> 6));

  // the lane's best value and the first chunk that has it
  float own = -__builtin_inff();
  int own_at = 0;
  over_chunks(row, wave, 0, row.per, [&](int c, const uint4& q) {
    float m = row.raw(q, 0);
#pragma unroll
    for (int e = 1; e < Row<F32>::E; ++e) m = fmaxf(m, row.raw(q, e));  // (not NaN, if there is another)
    own_at = m > own ? c : own_at;
    own = m > own ? m : own;
  });
  float top = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) s.top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < WAVES; ++v) top = fmaxf(top, s.top[v]);
  top = uni(top + 0.0f);
  auto answer = [&](int token, float prob) {
    p.token[t] = token;
    if (p.prob) p.prob[t] = prob;
  };
  const float temp = p.temperature ? p.temperature[t] : 1.0f;
  if (top == -__builtin_inff()) {
    if (threadIdx.x == 0) answer(-1, 0.0f);
    return;
  }
  if (!(temp > 0.0f)) {
    if (threadIdx.x == 0) s.n = ~0u;
    __syncthreads();
    if (own == top) atomicMin(&s.n, uint32_t(own_at));
    __syncthreads();
    if (own != top || s.n != uint32_t(own_at)) return;
    const uint4 q = row.load(own_at);
#pragma unroll
    for (int e = Row<F32>::E - 1; e >= 0; --e) own_at = row.raw(q, e) == top ? row.first(int(s.n)) + e : own_at;
    answer(own_at, 1.0f);
    return;
  }
  Weigh w;
  w.endless = top == __builtin_inff();
  w.top = w.endless ? 0.0f : top;
  w.lead = kPower[0];
  w.magic = 0x1.8p52 + double(p.sh);
  w.per_t = uni(fmax(1.4426950408889634 / double(temp), 1e-300));  // (not 0 where the temperature is infinite)
  w.least = uni(-1000.0 / w.per_t);
  // the last bin begins at (sh + 1.98) ln 2, where weights round to 0
  w.bins = uni(fminf(float(BINS) / (float(p.sh + 2) * 0.6931472f) / temp, 3e38f));
  w.width = uni(1.0f / w.bins);
  const int k_in = p.top_k ? p.top_k[t] : 0;
  const uint32_t k = k_in > 0 && k_in < p.V ? uint32_t(k_in) : 0u;
  const float top_p = p.top_p ? p.top_p[t] : 1.0f;
  const float min_p = p.min_p ? p.min_p[t] : 0.0f;
  const u64 least = uni(min_p > 0.0f ? u64(ceil(ldexp(fmin(double(min_p), 1.0), p.sh))) : u64(0));

  // By min_p few tokens stay, and they are gathered right away (with the weights' sum over the row, where top-p asks
  // for it): rows of 131072 with top-p 115-138 us, so 50.  The lanes that have one say about how many there are: of
  // 1024 tokens anywhere six in ten lanes.
  bool listed = false;
  if (least && !w.endless && (!k || (k > ENOUGH && !(top_p < 1.0f)))) {
    const float at = w.top + __builtin_amdgcn_logf(fminf(min_p, 1.0f)) / float(w.per_t);
    const float from = w.floor_of(std::min(w.bin(at), BINS - 2));
    if (__syncthreads_count(own >= from) <= THREADS / 2) {
      gather(s, row, w, from, [](float) { return true; });
      listed = uni(s.n) <= CAP;
    }
  }

  int last_bin = BINS;     // tokens of bins below it are kept,
  u64 last = ~u64(0);      // of its own those up to this place
  if (!listed && (k || top_p < 1.0f)) {
    u64 total = 0, m0 = 0;
    uint32_t c0 = 0;
    // The k-th best of the lanes' best values is one that k tokens reach at least, and few more: with top-k they
    // hold the answer, and no histogram of the row is needed.
    if (k && k <= ENOUGH) {
      clear_bins(s);
      own = clean(w.seen(own));
      const int b = w.bin(own);
      if (b < BINS - 1) atomicAdd(&s.count[b], 1u);
      if (threadIdx.x == 0) s.hi = 0;
      __syncthreads();
      const Before r = bins_before<false>(s, total);
      if (r.all_c >= k) {
        const int end = bin_of_cut(s, r, Cut{false, k, 0}, c0, m0);
        if (b <= end) atomicMax(&s.hi, key_of(own));
        __syncthreads();
        gather(s, row, w, uni(value_of(s.hi)), [](float) { return true; });
        if (answer_of_list(s, w, k, top_p, least, total, false, p.u[t], answer)) return;
      }
    }
    Before r = histogram(s, row, w, total);
    if (!k) {  // a nucleus of few tokens
      const int end = bin_of_cut(s, r, Cut{true, 0, border_of(top_p, total)}, c0, m0);
      if (c0 + s.count[end] <= CAP) {
        gather(s, row, w, w.floor_of(end), [&](float x) { return w.bin(x) <= end; });
        if (answer_of_list(s, w, k, top_p, least, total, false, p.u[t], answer)) return;
      }
    }
    u64 kept = total;  // sum of the top k
    bool both = false;
    if (k) {
      const int end = bin_of_cut(s, r, Cut{false, k, 0}, c0, m0);
      const uint32_t n = s.count[end];
      kept = m0 + s.mass[end];
      last_bin = end;
      __syncthreads();
      if (top_p < 1.0f && c0 + n > k) {
        // The bin in which the nucleus of the top k ends is known before their sum is, nearly always: both bins'
        // tokens are gathered at once, one pass of 22 us less over a row of 131072.
        uint32_t c1;
        u64 m1;
        const int pb = bin_of_cut(s, r, Cut{true, 0, border_of(top_p, m0)}, c1, m1);
        const uint32_t np = s.count[pb];
        const u64 mp = s.mass[pb];
        both = pb < end && np + n <= CAP && border_of(top_p, kept) <= m1 + mp;
        if (both) {
          gather(s, row, w, w.floor_of(end), [&](float x) { return w.bin(x) == pb || w.bin(x) == end; });
          if (threadIdx.x < 2) s.found[threadIdx.x] = 0;
          const Token g = rank_list(s, w, np + n);
          const bool first = g.is && g.part == 0;
          if (first && g.rank >= np && g.rank - np < k - c0) atomicMax(&s.found[1], g.before + g.mine - mp);
          __syncthreads();
          const u64 border = border_of(top_p, m0 + s.found[1]) - m1;
          if (first && g.rank < np && g.before < border) atomicMax(&s.found[0], g.place);
          __syncthreads();
          last = s.found[0];
          last_bin = pb;
        }
      }
      if (!both && c0 + n > k) {
        u64 m;
        last = cut_bin(s, row, w, end, n, Cut{false, k - c0, 0}, m);
        kept = m0 + m;
        if (top_p < 1.0f && n > CAP) r = histogram(s, row, w, total);  // the bins were used
      }
    }
    if (top_p < 1.0f && !both) {
      const u64 border = border_of(top_p, kept);
      u64 m;
      const int pb = bin_of_cut(s, r, Cut{true, 0, border}, c0, m0);
      const u64 at = cut_bin(s, row, w, pb, s.count[pb], Cut{true, 0, border - m0}, m);
      last = pb < last_bin ? at : min(last, at);
      last_bin = pb;
    }
  }

  // the indices in whose share of the sum the target falls: a wavefront's, a few of its chunk groups, one
  last = uni(last);
  last_bin = uni(last_bin);
  const float from = last_bin < BINS ? w.floor_of(last_bin) : -__builtin_inff();
  const float chunks_from = w.endless ? __builtin_inff() : from;
  auto weight = [&](float x, int i) -> u64 {
    x = w.seen(x);
    bool stays = true;
    if (last_bin < BINS) {
      const int b = w.bin(x);
      stays = x >= from && b <= last_bin;
      if (__any(stays && b == last_bin)) stays = stays && (b < last_bin || place_of(clean(x), i) <= last);
      if (!__any(stays)) return 0;
    }
    u64 v = w(x);
    if (least) v = v >= least ? v : 0;
    return stays ? v : 0;
  };
  // nearly all rows keep the tokens up to one of them in order
  const bool simple = !w.endless && (listed || !least) && (last_bin == BINS || last != ~u64(0));
  const float end_x = last_bin < BINS ? value_of(uint32_t(last >> 32)) : -__builtin_inff();
  const int end_i = last_bin < BINS ? int(uint32_t(last)) : 0x7FFFFFFF;
  auto sum_of = [&](int of, int i0, int i1) {
    if (simple) return mass_upto(row, w, of, i0, i1, end_x, end_i);
    u64 sum = 0;
    over_part(row, of, i0, i1, chunks_from, [&](float x, int i) { sum += weight(x, i); });
    return sum;
  };
  u64 all = 0, left = 0;
  int of = 0, at0 = 0, n = WAVES * row.per;  // chunk groups at0 .. at0 + n of wavefront `of` (first: of all)
  for (bool first = true; first || n > 1; first = false) {
    const int each = first ? row.per : (n + WAVES - 1) / WAVES;
    const int i0 = first ? 0 : at0 + std::min(wave * each, n), i1 = first ? row.per : at0 + std::min((wave + 1) * each, n);
    const u64 sum = listed && !(top_p < 1.0f) ? 0 : wave_sum(sum_of(first ? wave : of, i0, i1));
    if (first) {
      block_before(s, lane ? 0 : sum, all);
      if (listed) {
        answer_of_list(s, w, k, top_p, least, all, true, p.u[t], answer);
        return;
      }
      left = part_of(p.u[t], all);
    }
    const int v = pick(s, sum, left, left);
    if (first) {
      of = v;
      n = row.per;
    } else {
      at0 += v * each;
      n = std::min(n - v * each, each);
    }
  }
  if (wave) return;
  u64 mine = 0;
  over_part(row, of, at0, at0 + 1, chunks_from, [&](float x, int i) { mine += weight(x, i); });
  u64 at = wave_upto(mine) - mine;
  over_part(row, of, at0, at0 + 1, chunks_from, [&](float x, int i) {
    const u64 v = weight(x, i);
    if (at <= left && left < at + v) answer(i, float(double(v) / double(all)));
    at += v;
  });
}

}  // namespace

size_t sample_ws(int64_t, int64_t) { return 0; }

hipError_t launch_sample(SampleLaunch p, hipStream_t st) {
  p.sh = 62;
  for (int64_t v = 1; v < p.V; v <<= 1) --p.sh;
  p.sh = std::min(p.sh, 51);  // weights below 2^52
  if (p.x_dtype == F32)
    sample_kernel<true><<<grid_of(p.T), THREADS, 0, st>>>(p);
  else
    sample_kernel<false><<<grid_of(p.T), THREADS, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace uq
