// The paged key/value cache: new rows written (rotated, quantized) and ranges
// of positions read back.  Layout, quantiser and errors in uniquan.h.
//
// 16 lanes take one head of one row; lane l holds its channels l + 16 c, so a
// rotary pair (i, i + d/2) is in one lane and a group of 32 channels is two
// values of each of the 16 lanes.
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

__device__ __forceinline__ uint16_t to_bf16(float x) { return uint16_t(pack_bf16x2(x, x)); }

// Minimum, maximum and whether all values are finite, over 16 lanes.
struct Span {
  float lo, hi;
  bool fine;
};
__device__ __forceinline__ Span span16(Span s) {
#pragma unroll
  for (int m = 8; m >= 1; m >>= 1) {
    s.lo = fminf(s.lo, __shfl_xor(s.lo, m));
    s.hi = fmaxf(s.hi, __shfl_xor(s.hi, m));
    s.fine = bool(__shfl_xor(int(s.fine), m)) && s.fine;
  }
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

enum Kind : int { Q_HEAD = 0, K_HEAD = 1, V_HEAD = 2 };

template <int D>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendLaunch p) {
  constexpr int N = D / 16;
  const KvCache& c = p.c;
  const int l = threadIdx.x & 15;
  const int heads = (p.q ? p.H : 0) + 2 * c.H_kv;
  const int64_t vec = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4);
  const int64_t t = vec / heads;
  if (t >= p.T) return;
  int h = int(vec % heads);
  int kind = V_HEAD;
  const int n_q = p.q ? p.H : 0;
  if (h < n_q) {
    kind = Q_HEAD;
  } else if (h < n_q + c.H_kv) {
    kind = K_HEAD;
    h -= n_q;
  } else {
    h -= n_q + c.H_kv;
  }
  const int pos = p.pos[t];
  const int64_t s = p.seq ? p.seq[t] : t;
  if (pos < 0 || pos >= c.max_pages << c.log_page || (p.cs && pos >= p.n_cs) || s < 0 || s >= c.n_seq) return;

  const bool f32 = p.in_dtype == F32;
  const void* src = kind == Q_HEAD ? p.q : kind == K_HEAD ? p.k : p.v;
  const int64_t off = t * (kind == Q_HEAD ? p.ld_q : kind == K_HEAD ? p.ld_k : p.ld_v) + int64_t(h) * D;
  float x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = load1(src, off + l + 16 * i, f32);
  if (kind != V_HEAD && p.cs) {
    const float2* cs = reinterpret_cast<const float2*>(p.cs) + int64_t(pos) * (D / 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 a = cs[l + 16 * i];
      const float x1 = x[i], x2 = x[i + N / 2];
      x[i] = x1 * a.x - x2 * a.y;
      x[i + N / 2] = x2 * a.x + x1 * a.y;
    }
  }
  if (kind == Q_HEAD) {
    uint16_t* o = p.q_out + (t * p.H + h) * D;
#pragma unroll
    for (int i = 0; i < N; ++i) o[l + 16 * i] = to_bf16(x[i]);
    return;
  }
  const int page = kv_page(c, s, pos);
  if (page < 0) return;
  const int place = pos & (c.page_len - 1);
  const int64_t ph = int64_t(page) * c.H_kv + h;
  const int64_t row = ph * c.page_len + place;
  if (c.format == KV_BF16) {
    uint16_t* o = static_cast<uint16_t*>(kind == K_HEAD ? c.k : c.v) + row * D;
#pragma unroll
    for (int i = 0; i < N; ++i) o[l + 16 * i] = to_bf16(x[i]);
    return;
  }
  const float top = c.format == KV_U8 ? 255.0f : 15.0f;
  const int per = c.group / 16;  // values of a lane in one group: 2 or N
  uint32_t* stat = reinterpret_cast<uint32_t*>(kind == K_HEAD ? c.k_stat : c.v_stat);
  uint8_t* o = static_cast<uint8_t*>(kind == K_HEAD ? c.k : c.v) + row * (c.format == KV_U8 ? D : D / 2);
  uint32_t code[N];
  Span all{x[0], x[0], true};
  Quant q;
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    Span sp{fminf(x[i], x[i + 1]), fmaxf(x[i], x[i + 1]), x[i] - x[i] == 0.0f && x[i + 1] - x[i + 1] == 0.0f};
    sp = span16(sp);
    if (per == 2) {
      q = quant_of(sp, top);
      code[i] = code_of(x[i], q, top);
      code[i + 1] = code_of(x[i + 1], q, top);
      if (l == 0) stat[(ph * (D / 32) + i / 2) * c.page_len + place] = pack_bf16x2(q.scale, q.lo);
    }
    all = Span{fminf(all.lo, sp.lo), fmaxf(all.hi, sp.hi), all.fine && sp.fine};
  }
  if (per != 2) {
    q = quant_of(all, top);
#pragma unroll
    for (int i = 0; i < N; ++i) code[i] = code_of(x[i], q, top);
    if (l == 0) stat[ph * c.page_len + place] = pack_bf16x2(q.scale, q.lo);
  }
  if (kind == K_HEAD) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int ch = l + 16 * i, run = (ch / 8 % 4) * (D / 4) + 8 * (ch / 32);
      if (c.format == KV_U8) {
        o[run + ch % 8] = uint8_t(code[i]);
      } else {  // channels j and j + 2 of a run of eight share a byte
        const uint32_t other = uint32_t(__shfl_xor(int(code[i]), 2));
        if ((l & 2) == 0) o[(run + (ch % 8) / 2 + 4 * (ch % 2)) / 2] = uint8_t(code[i] | other << 4);
      }
    }
  } else if (c.format == KV_U8) {
#pragma unroll
    for (int i = 0; i < N; ++i) o[l * N + i] = uint8_t(code[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) o[(l * N + i) / 2] = uint8_t(code[i] | code[i + 1] << 4);
  }
}

// Value of channel ch at a cache row.
template <int D>
__device__ __forceinline__ float kv_value(const KvCache& c, bool key, int64_t ph, int place, int ch) {
  const int64_t row = ph * c.page_len + place;
  const void* base = key ? c.k : c.v;
  if (c.format == KV_BF16) return bf16_to_f32(static_cast<const uint16_t*>(base)[row * D + ch]);
  const bool u8 = c.format == KV_U8;
  int at;
  if (key)
    at = (ch / 8 % 4) * (D / 4) + 8 * (ch / 32) + (u8 ? ch % 8 : (ch % 8) / 2 + 4 * (ch % 2));
  else
    at = (ch % 16) * (D / 16) + ch / 16;
  const uint8_t* o = static_cast<const uint8_t*>(base) + row * (u8 ? D : D / 2);
  const uint32_t code = u8 ? o[at] : o[at / 2] >> (4 * (at & 1)) & 15u;
  const uint32_t st = reinterpret_cast<const uint32_t*>(key ? c.k_stat : c.v_stat)[
      (ph * (D / c.group) + ch / c.group) * c.page_len + place];
  const float scale = __uint_as_float(st << 16), lo = __uint_as_float(st & 0xFFFF0000u);
  return lo + scale * float(code);
}

template <int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadLaunch p) {
  const KvCache& c = p.c;
  const int l = threadIdx.x & 15;
  const int64_t vec = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4);  // (h, s, i)
  if (vec >= c.H_kv * c.n_seq * p.L) return;
  const int64_t i = vec % p.L, s = vec / p.L % c.n_seq;
  const int h = int(vec / p.L / c.n_seq);
  const int64_t pos = i + (p.start ? p.start[s] : 0);
  int page = -1;
  if (pos >= 0 && pos < p.lens[s] && pos < c.max_pages << c.log_page) page = kv_page(c, s, int(pos));
  for (int side = 0; side < 2; ++side) {
    void* out = side ? p.V : p.K;
    if (!out) continue;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      const int ch = l + 16 * e;
      const float x = page < 0 ? 0.0f
                               : kv_value<D>(c, side == 0, int64_t(page) * c.H_kv + h, int(pos) & (c.page_len - 1), ch);
      if (p.out_dtype == F32)
        static_cast<float*>(out)[vec * D + ch] = x;
      else
        static_cast<uint16_t*>(out)[vec * D + ch] = to_bf16(x);
    }
  }
}

}  // namespace

hipError_t launch_kv_append(const KvAppendLaunch& p, hipStream_t st) {
  const int64_t n = p.T * ((p.q ? p.H : 0) + 2 * p.c.H_kv);
  const dim3 grid{unsigned((n + 15) / 16)};
  if (p.c.d == 128)
    kv_append_kernel<128><<<grid, 256, 0, st>>>(p);
  else
    kv_append_kernel<64><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvReadLaunch& p, hipStream_t st) {
  const int64_t n = p.c.H_kv * p.c.n_seq * p.L;
  const dim3 grid{unsigned((n + 15) / 16)};
  if (p.c.d == 128)
    kv_read_kernel<128><<<grid, 256, 0, st>>>(p);
  else
    kv_read_kernel<64><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace uq
