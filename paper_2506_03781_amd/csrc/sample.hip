// One token per row of logits (uniquan_sample); definition and errors in
// uniquan.h.
//
// Weights.  w = rint(2^sh e^((x - max) / t)), sh = 62 - ceil(log2 V): integers
// whose sums are exact and the same in any order, so that every comparison of
// a running sum with a border has one answer however the work is split.  The
// exponential is taken in 64 bits: with one in 32 bits the running sums of some
// ten thousand tokens are off by 1e-7 of their total, and a random number
// falls that near to one of the borders once in some hundred rows.
//
// A workgroup takes a row and reads it once per pass (the first time from
// memory, then from the caches):
//   maximum    of (value, lowest index): also the greedy answer.
//   histogram  counts and sums of weights in BINS equal steps of (max - x) / t,
//              where top-k or top-p is on.  Its running sums say in which bin
//              the k-th token lies and in which the nucleus ends.
//   gather     what lies up to there, if it is at most CAP tokens, goes to LDS
//              and everything else happens there (sorted by value, cut, sorted by
//              index); else the bin in which the cut lies, to find it exactly.
//              A bin of more than CAP tokens is cut by further histograms, of
//              equal steps between its smallest and largest value; many tokens of
//              one value by their indices.
//   sums       of the weights kept, per run of indices of a wavefront; the run in
//              which u times the total falls is read again by one wavefront.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "uq_device.h"
#include "uq_launch.h"

namespace uq {

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int BINS = 2048;  // two a thread
constexpr int CAP = 4096;   // tokens that are sorted in LDS
constexpr int RUNS = 1024;  // runs of indices

typedef unsigned long long u64;

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

__device__ __forceinline__ u64 shfl_up(u64 x, int d) {
  return u64(__shfl_up(uint32_t(x >> 32), d)) << 32 | __shfl_up(uint32_t(x), d);
}
__device__ __forceinline__ u64 shfl_xor(u64 x, int d) {
  return u64(__shfl_xor(uint32_t(x >> 32), d)) << 32 | __shfl_xor(uint32_t(x), d);
}
__device__ __forceinline__ u64 shfl(u64 x, int l) {
  return u64(__shfl(uint32_t(x >> 32), l)) << 32 | __shfl(uint32_t(x), l);
}
__device__ __forceinline__ u64 wave_sum(u64 x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += shfl_xor(x, d);
  return x;
}
// Sum over the lanes up to this one.
__device__ __forceinline__ u64 wave_upto(u64 x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 y = shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  return x;
}

struct Lds {
  u64 mass[BINS];
  uint32_t count[BINS];
  u64 list[CAP];
  u64 wave[WAVES];
  u64 found[4];
  uint32_t n, lo, hi;
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

// A row as aligned chunks of 16 bytes, the first and the last in part.
template <bool F32>
struct Row {
  static constexpr int E = F32 ? 4 : 8;
  const char* at;  // of chunk 0
  int shift;       // elements of chunk 0 before the row
  int V, chunks;

  __device__ Row(const void* x, int64_t off, int V) : V(V) {
    const char* p = static_cast<const char*>(x) + off * (F32 ? 4 : 2);
    const int over = int(reinterpret_cast<uintptr_t>(p) & 15);
    at = p - over;
    shift = over / (F32 ? 4 : 2);
    chunks = (shift + V + E - 1) / E;
  }
  __device__ __forceinline__ int first(int c) const { return c * E - shift; }
  __device__ __forceinline__ bool whole(int c) const { return first(c) >= 0 && first(c) + E <= V; }
  // Words of chunk c; what is outside the row is -infinity.
  __device__ __forceinline__ uint4 load(int c) const {
    if (whole(c)) return reinterpret_cast<const uint4*>(at)[c];
    uint32_t w[4] = {};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = first(c) + e;
      const bool in = i >= 0 && i < V;
      if constexpr (F32) {
        w[e] = in ? reinterpret_cast<const uint32_t*>(at)[int64_t(c) * E + e] : 0xFF800000u;
      } else {
        w[e / 2] |= uint32_t(in ? reinterpret_cast<const uint16_t*>(at)[int64_t(c) * E + e] : 0xFF80u) << (16 * (e & 1));
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  // Element e of a chunk; NaN as -infinity, -0 as 0.
  static __device__ __forceinline__ float value(const uint4& c, int e) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    const float x = F32 ? __uint_as_float(w[e]) : __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    return x == x ? x + 0.0f : -__builtin_inff();
  }
};

// f(chunk, its words) for every chunk of the row, thread by thread; the wavefront
// stays together (chunks behind the end are -infinity).
template <bool F32, typename Fn>
__device__ __forceinline__ void over_row(const Row<F32>& r, Fn f) {
  constexpr int AHEAD = 4;
  for (int c0 = threadIdx.x; c0 - int(threadIdx.x & 63) < r.chunks; c0 += AHEAD * THREADS) {
    uint4 w[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) w[a] = r.load(c0 + a * THREADS);
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
      if (c0 + a * THREADS - int(threadIdx.x & 63) < r.chunks) f(c0 + a * THREADS, w[a]);
  }
}

struct Weigh {
  float top;       // the row's maximum
  double inv_t;    // 1 / temperature
  float bins;      // bins per unit of max - x
  int sh;

  // Monotone in x; weights in the last bin are 0.
  __device__ __forceinline__ int bin(float x) const {
    if (x == top) return 0;
    const float z = (top - x) * bins;
    return z < float(BINS - 1) ? int(z) : BINS - 1;
  }
  __device__ __forceinline__ u64 operator()(float x) const {
    if (x == top) return u64(1) << sh;
    const double y = (double(x) - double(top)) * inv_t;
    if (!(y > -0.6931472 * (sh + 2))) return 0;  // also x = -infinity
    return u64(rint(ldexp(exp(y), sh)));
  }
};

// Sorts list[0, n) ascending, n <= CAP; what is behind up to the next power of two is overwritten.
__device__ void sort_list(Lds& s, int n) {
  int m = 64;
  while (m < n) m <<= 1;
  for (int i = n + threadIdx.x; i < m; i += THREADS) s.list[i] = ~u64(0);
  __syncthreads();
  for (int k = 2; k <= m; k <<= 1) {
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int t = threadIdx.x; t < m / 2; t += THREADS) {
        const int i = (t & ~(j - 1)) << 1 | (t & (j - 1));
        const u64 a = s.list[i], b = s.list[i + j];
        if ((a > b) == ((i & k) == 0)) {
          s.list[i] = b;
          s.list[i + j] = a;
        }
      }
      __syncthreads();
    }
  }
}

// A cut in the order of the tokens: the first `count` of them, or, where by_mass,
// those before which the weights sum to less than `mass`.
struct Cut {
  bool by_mass;
  uint32_t count;
  u64 mass;
};

// Running sums of the histogram before each thread's bins 2 i and 2 i + 1.
struct Before {
  uint32_t c[2];
  u64 m[2];
};
__device__ __forceinline__ Before bins_before(Lds& s, u64& all) {
  const int b = 2 * threadIdx.x;
  u64 nc;
  const u64 m0 = s.mass[b], m1 = s.mass[b + 1];
  const uint32_t c0 = s.count[b], c1 = s.count[b + 1];
  Before r;
  r.m[0] = block_before(s, m0 + m1, all);
  r.m[1] = r.m[0] + m0;
  r.c[0] = uint32_t(block_before(s, u64(c0) + c1, nc));
  r.c[1] = r.c[0] + c0;
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

// The bin in which the cut lies; sums before it. Bins behind the last token's do not count.
__device__ __forceinline__ int bin_of_cut(Lds& s, const Before& r, const Cut& cut, uint32_t& c, u64& m) {
  if (threadIdx.x == 0) s.found[0] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int b = 2 * threadIdx.x + i;
    const bool starts = s.count[b] > 0 && (cut.by_mass ? r.m[i] < cut.mass : r.c[i] < cut.count);
    if (starts) atomicMax(&s.found[0], u64(b));
  }
  __syncthreads();
  const int b = int(s.found[0]);
  if (threadIdx.x == unsigned(b / 2)) {
    s.found[1] = b & 1 ? r.c[1] : r.c[0];
    s.found[2] = b & 1 ? r.m[1] : r.m[0];
  }
  __syncthreads();
  c = uint32_t(s.found[1]);
  m = s.found[2];
  __syncthreads();
  return b;
}

// The cut among the tokens of bin b (n of them): place of the last one before it, and the sum of the weights there.
template <bool F32>
__device__ u64 cut_bin(Lds& s, const Row<F32>& row, const Weigh& w, int b, uint32_t n, Cut cut, u64& mass) {
  uint32_t lo = 0, hi = ~0u;  // keys still in question
  mass = 0;
  while (n > CAP) {
    __syncthreads();
    if (threadIdx.x == 0) {
      s.lo = ~0u;
      s.hi = 0;
    }
    __syncthreads();
    uint32_t a = ~0u, z = 0;
    over_row(row, [&](int, const uint4& c) {
#pragma unroll
      for (int e = 0; e < Row<F32>::E; ++e) {
        const float x = row.value(c, e);
        const uint32_t k = key_of(x);
        if (w.bin(x) == b && k >= lo && k <= hi) {
          a = min(a, k);
          z = max(z, k);
        }
      }
    });
    atomicMin(&s.lo, a);
    atomicMax(&s.hi, z);
    __syncthreads();
    lo = s.lo;
    hi = s.hi;
    if (lo == hi) break;
    clear_bins(s);
    const u64 span = u64(hi) - lo + 1;
    auto sub = [&](uint32_t k) { return int((u64(k - lo) * BINS) / span); };
    over_row(row, [&](int, const uint4& c) {
#pragma unroll
      for (int e = 0; e < Row<F32>::E; ++e) {
        const float x = row.value(c, e);
        const uint32_t k = key_of(x);
        if (w.bin(x) == b && k >= lo && k <= hi) {
          atomicAdd(&s.count[sub(k)], 1u);
          atomicAdd(&s.mass[sub(k)], w(x));
        }
      }
    });
    __syncthreads();
    u64 all;
    const Before r = bins_before(s, all);
    uint32_t c;
    u64 m;
    const int v = bin_of_cut(s, r, cut, c, m);
    n = s.count[v];
    cut.count -= cut.by_mass ? 0 : c;
    cut.mass -= cut.by_mass ? m : 0;
    mass += m;
    // keys k with sub(k) == v
    const u64 k0 = (u64(v) * span + BINS - 1) / BINS, k1 = (u64(v + 1) * span + BINS - 1) / BINS;
    hi = uint32_t(lo + k1 - 1);
    lo = uint32_t(lo + k0);
  }
  __syncthreads();
  if (n > CAP) {  // one value: the first r of them by index
    const u64 one = w(value_of(lo));
    u64 r = cut.by_mass ? (one ? (cut.mass + one - 1) / one : n) : cut.count;
    r = r < n ? r : n;
    mass += r * one;
    if (r == n) return ~u64(0);
    // how many lie in each run of indices
    const int per = (row.chunks + RUNS - 1) / RUNS;
    for (int i = threadIdx.x; i < RUNS; i += THREADS) s.count[i] = 0;
    __syncthreads();
    over_row(row, [&](int c, const uint4& q) {
      uint32_t k = 0;
#pragma unroll
      for (int e = 0; e < Row<F32>::E; ++e) k += key_of(row.value(q, e)) == lo;
      if (k && c < row.chunks) atomicAdd(&s.count[c / per], k);
    });
    __syncthreads();
    u64 all;
    const u64 mine = s.count[threadIdx.x], before = block_before(s, mine, all);
    if (before < r && r <= before + mine) {  // one thread: r >= 1
      u64 left = r - before;
      u64 at = 0;
      for (int c = threadIdx.x * per; c < row.chunks && left; ++c) {
        const uint4 q = row.load(c);
#pragma unroll
        for (int e = 0; e < Row<F32>::E; ++e)
          if (left && key_of(row.value(q, e)) == lo) {
            --left;
            at = u64(row.first(c) + e);
          }
      }
      s.found[3] = u64(lo) << 32 | at;
    }
    __syncthreads();
    return s.found[3];
  }
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  over_row(row, [&](int c, const uint4& q) {
#pragma unroll
    for (int e = 0; e < Row<F32>::E; ++e) {
      const float x = row.value(q, e);
      const uint32_t k = key_of(x);
      const int i = row.first(c) + e;
      if (i >= 0 && i < row.V && w.bin(x) == b && k >= lo && k <= hi) s.list[atomicAdd(&s.n, 1u) & (CAP - 1)] = u64(k) << 32 | uint32_t(i);
    }
  });
  __syncthreads();
  sort_list(s, n);
  u64 v[CAP / THREADS], sum = 0, all;
#pragma unroll
  for (int i = 0; i < CAP / THREADS; ++i) {
    const uint32_t at = threadIdx.x * (CAP / THREADS) + i;
    v[i] = at < n ? w(value_of(uint32_t(s.list[at] >> 32))) : 0;
    sum += v[i];
  }
  u64 before = block_before(s, sum, all);
  if (threadIdx.x == 0) s.found[0] = s.found[1] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < CAP / THREADS; ++i) {
    const uint32_t at = threadIdx.x * (CAP / THREADS) + i;
    if (at < n && (cut.by_mass ? before < cut.mass : at < cut.count)) {
      atomicMax(&s.found[0], u64(at) + 1);
      atomicMax(&s.found[1], before + v[i]);
    }
    before += v[i];
  }
  __syncthreads();
  const u64 kept = s.found[0];
  mass += s.found[1];
  return kept ? s.list[kept - 1] : 0;
}

// Counts and sums of weights per bin, and the sums before each thread's bins.
template <bool F32>
__device__ __forceinline__ Before histogram(Lds& s, const Row<F32>& row, const Weigh& w, u64& total) {
  clear_bins(s);
  over_row(row, [&](int, const uint4& q) {
#pragma unroll
    for (int e = 0; e < Row<F32>::E; ++e) {
      const float x = row.value(q, e);
      const int b = w.bin(x);
      if (b < BINS - 1) {  // not what is outside the row
        atomicAdd(&s.count[b], 1u);
        atomicAdd(&s.mass[b], w(x));
      }
    }
  });
  __syncthreads();
  return bins_before(s, total);
}

// floor(u total) for u in [0, 1); the last unit from 1 on.
__device__ __forceinline__ u64 part_of(float u, u64 total) {
  if (!(u > 0.0f)) return 0;
  if (u >= 1.0f) return total - 1;
  return __umul64hi(u64(double(u) * 0x1p64), total);
}

// Whether sums below it are below p total, p < 1: ceil(p total).
__device__ __forceinline__ u64 border_of(float p, u64 total) {
  if (!(p > 0.0f)) return 1;  // the first token
  const u64 f = u64(double(p) * 0x1p64), hi = __umul64hi(f, total), lo = f * total;
  return hi + (lo != 0);
}

template <bool F32>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleLaunch p) {
  __shared__ Lds s;
  const int64_t t = blockIdx.x;
  const Row<F32> row(p.x, t * p.ld, p.V);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  u64 best = ~u64(0);
  over_row(row, [&](int c, const uint4& q) {
#pragma unroll
    for (int e = 0; e < Row<F32>::E; ++e) {
      const float x = row.value(q, e);
      const u64 at = place_of(x, row.first(c) + e);
      best = x > -__builtin_inff() && at < best ? at : best;
    }
  });
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) best = min(best, shfl_xor(best, d));
  if (lane == 0) s.wave[wave] = best;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < WAVES; ++v) best = min(best, s.wave[v]);
  auto answer = [&](int token, float prob) {
    p.token[t] = token;
    if (p.prob) p.prob[t] = prob;
  };
  const float temp = p.temperature ? p.temperature[t] : 1.0f;
  if (best == ~u64(0) || !(temp > 0.0f)) {
    if (threadIdx.x == 0) answer(best == ~u64(0) ? -1 : int(uint32_t(best)), best == ~u64(0) ? 0.0f : 1.0f);
    return;
  }
  Weigh w;
  w.top = value_of(uint32_t(best >> 32));
  w.inv_t = 1.0 / double(temp);
  w.sh = p.sh;
  // the last bin begins at (sh + 1.98) ln 2, where weights round to 0
  w.bins = fminf(float(BINS) / (float(p.sh + 2) * 0.6931472f) / temp, 3e38f);
  const int k_in = p.top_k ? p.top_k[t] : 0;
  const uint32_t k = k_in > 0 && k_in < p.V ? uint32_t(k_in) : 0u;
  const float top_p = p.top_p ? p.top_p[t] : 1.0f;
  const float min_p = p.min_p ? p.min_p[t] : 0.0f;
  const u64 least = min_p > 0.0f ? u64(ceil(ldexp(fmin(double(min_p), 1.0), p.sh))) : 0;

  int last_bin = BINS;     // tokens of bins below it are kept,
  u64 last = ~u64(0);      // of its own those up to this place
  if (k || top_p < 1.0f) {
    u64 total;
    Before r = histogram(s, row, w, total);
    uint32_t c0 = 0;
    u64 m0 = 0;
    int kb = BINS - 1, kb_of = 0;
    u64 kept = total;  // of the top k
    if (k) {
      kb = bin_of_cut(s, r, Cut{false, k, 0}, c0, m0);
      const uint32_t n = s.count[kb];
      last_bin = kb_of = kb;
      kept = m0 + s.mass[kb];
      if (c0 + n <= k) kb = BINS - 1;  // whole bins, the rest has no weight or none is left
    }
    // everything up to the end of the cut's bin in LDS?
    uint32_t cp = c0;
    u64 mp;
    const int end = k ? kb_of : bin_of_cut(s, r, Cut{true, 0, border_of(top_p, total)}, cp, mp);
    {
      const uint32_t upto = cp + s.count[end];
      if (upto <= CAP) {
        if (threadIdx.x == 0) s.n = 0;
        __syncthreads();
        over_row(row, [&](int c, const uint4& q) {
#pragma unroll
          for (int e = 0; e < Row<F32>::E; ++e) {
            const float x = row.value(q, e);
            const int i = row.first(c) + e;
            if (i >= 0 && i < row.V && w.bin(x) <= end) s.list[atomicAdd(&s.n, 1u) & (CAP - 1)] = place_of(x, i);
          }
        });
        __syncthreads();
        uint32_t n = upto;
        sort_list(s, n);
        if (k && k < n) n = k;
        u64 v[CAP / THREADS], sum = 0, all;
#pragma unroll
        for (int i = 0; i < CAP / THREADS; ++i) {
          const uint32_t at = threadIdx.x * (CAP / THREADS) + i;
          v[i] = at < n ? w(value_of(uint32_t(s.list[at] >> 32))) : 0;
          sum += v[i];
        }
        u64 before = block_before(s, sum, all);
        if (!k) all = total;
        const u64 border = top_p < 1.0f ? border_of(top_p, all) : ~u64(0);
        if (threadIdx.x == 0) s.found[0] = 0;
        __syncthreads();
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < CAP / THREADS; ++i) {
          const uint32_t at = threadIdx.x * (CAP / THREADS) + i;
          if (at < n && before < border && v[i] >= least) mine = at + 1;
          before += v[i];
        }
        if (mine) atomicMax(&s.found[0], u64(mine));
        __syncthreads();
        n = uint32_t(s.found[0]);
        // by index: (index, key)
        for (uint32_t i = threadIdx.x; i < n; i += THREADS) s.list[i] = s.list[i] << 32 | s.list[i] >> 32;
        sort_list(s, n);
        sum = 0;
#pragma unroll
        for (int i = 0; i < CAP / THREADS; ++i) {
          const uint32_t at = threadIdx.x * (CAP / THREADS) + i;
          v[i] = at < n ? w(value_of(uint32_t(s.list[at]))) : 0;
          sum += v[i];
        }
        before = block_before(s, sum, all);
        const u64 target = part_of(p.u[t], all);
#pragma unroll
        for (int i = 0; i < CAP / THREADS; ++i) {
          const uint32_t at = threadIdx.x * (CAP / THREADS) + i;
          if (before <= target && target < before + v[i])
            answer(int(uint32_t(s.list[at] >> 32)), float(double(v[i]) / double(all)));
          before += v[i];
        }
        return;
      }
    }
    bool stale = false;  // the histogram was used for another
    if (kb < BINS - 1) {
      const uint32_t n = s.count[kb];
      stale = n > CAP;
      u64 m;
      last = cut_bin(s, row, w, kb, n, Cut{false, k - c0, 0}, m);
      kept = m0 + m;
    }
    if (top_p < 1.0f) {
      if (stale) r = histogram(s, row, w, total);
      const u64 border = border_of(top_p, kept);
      const int pb = bin_of_cut(s, r, Cut{true, 0, border}, cp, mp);
      u64 m;
      const u64 end = cut_bin(s, row, w, pb, s.count[pb], Cut{true, 0, border - mp}, m);
      last = pb < last_bin ? end : min(last, end);
      last_bin = pb;
    }
  }

  // sums of the kept weights per run of indices
  const int pieces = (row.chunks + 63) / 64;  // of a wavefront's chunks
  const int per = (pieces + RUNS - 1) / RUNS;
  auto weight = [&](float x, int i) -> u64 {
    if (i < 0 || i >= row.V) return 0;
    const u64 v = w(x);
    const int b = w.bin(x);
    return v >= least && (b < last_bin || (b == last_bin && place_of(x, i) <= last)) ? v : 0;
  };
  __syncthreads();
  for (int i = threadIdx.x; i < RUNS; i += THREADS) s.mass[i] = 0;
  __syncthreads();
  over_row(row, [&](int c, const uint4& q) {
    u64 sum = 0;
#pragma unroll
    for (int e = 0; e < Row<F32>::E; ++e) sum += weight(row.value(q, e), row.first(c) + e);
    sum = wave_sum(sum);
    if (lane == 0 && sum) atomicAdd(&s.mass[c / 64 / per], sum);
  });
  __syncthreads();
  u64 all;
  const u64 mine = s.mass[threadIdx.x], before = block_before(s, mine, all);
  const u64 target = part_of(p.u[t], all);
  if (before <= target && target < before + mine) {
    s.found[0] = threadIdx.x;
    s.found[1] = target - before;
  }
  __syncthreads();
  if (wave) return;
  u64 left = s.found[1];
  const int run = int(s.found[0]);
  for (int piece = run * per; piece < run * per + per; ++piece) {
    const int c = piece * 64 + lane;
    const uint4 q = row.load(c);
    u64 v[Row<F32>::E], sum = 0;
#pragma unroll
    for (int e = 0; e < Row<F32>::E; ++e) {
      v[e] = weight(row.value(q, e), row.first(c) + e);
      sum += v[e];
    }
    const u64 upto = wave_upto(sum), end = shfl(upto, 63);
    if (left >= end) {
      left -= end;
      continue;
    }
    u64 at = upto - sum;
#pragma unroll
    for (int e = 0; e < Row<F32>::E; ++e) {
      if (at <= left && left < at + v[e]) answer(row.first(c) + e, float(double(v[e]) / double(all)));
      at += v[e];
    }
    return;
  }
}

}  // namespace

size_t sample_ws(int64_t, int64_t) { return 0; }

hipError_t launch_sample(SampleLaunch p, hipStream_t st) {
  p.sh = 62;
  for (int64_t v = 1; v < p.V; v <<= 1) --p.sh;
  p.sh = std::min(p.sh, 52);
  if (p.x_dtype == F32)
    sample_kernel<true><<<unsigned(p.T), THREADS, 0, st>>>(p);
  else
    sample_kernel<false><<<unsigned(p.T), THREADS, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace uq
