// Attention of one new token per sequence over the paged key/value cache
// (uniquan_attn_decode).  One workgroup per sequence and query head; its four
// wavefronts take the positions in turn, a lane d / 64 channels, with a
// running maximum and sum, and are joined in LDS.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "uq_device.h"
#include "uq_kv.h"
#include "uq_launch.h"

namespace uq {

namespace {

constexpr float LOG2E_D = 1.44269504088896341f;
constexpr float NEG_INF = -__builtin_inff();

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
__global__ __launch_bounds__(256) void attn_decode_kernel(AttnDecodeLaunch p) {
  constexpr int N = D / 64;
  const KvCache& c = p.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t s = blockIdx.x / p.H;
  const int h = blockIdx.x % p.H, hk = h / (p.H / c.H_kv);
  const int64_t cap = c.max_pages << c.log_page;
  const int len = int(p.lens[s] < cap ? p.lens[s] : cap);
  float q[N], o[N] = {}, m = NEG_INF, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) q[i] = bf16_to_f32(p.Q[s * p.ld_q + int64_t(h) * D + lane + 64 * i]);
  for (int t = wave; t < len; t += 4) {
    const int page = kv_page(c, s, t);
    if (page < 0) continue;
    const int64_t ph = int64_t(page) * c.H_kv + hk;
    const int place = t & (c.page_len - 1);
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) x += q[i] * kv_value<D>(c, true, ph, place, lane + 64 * i);
#pragma unroll
    for (int k = 32; k >= 1; k >>= 1) x += __shfl_xor(x, k);
    x *= p.scale * LOG2E_D;
    const float m1 = fmaxf(m, x);
    const float ref = m1 == NEG_INF ? 0.0f : m1;
    const float e = __builtin_amdgcn_exp2f(x - ref), f = __builtin_amdgcn_exp2f(m - ref);
    m = m1;
    sum = sum * f + e;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * f + e * kv_value<D>(c, false, ph, place, lane + 64 * i);
  }
  __shared__ float so[4][D], sm[4], ss[4];
#pragma unroll
  for (int i = 0; i < N; ++i) so[wave][lane + 64 * i] = o[i];
  if (lane == 0) {
    sm[wave] = m;
    ss[wave] = sum;
  }
  __syncthreads();
  if (wave) return;
  float top = NEG_INF;
  for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w]);
  const float ref = top == NEG_INF ? 0.0f : top;
  float total = 0.0f;
  for (int w = 0; w < 4; ++w) total += ss[w] * __builtin_amdgcn_exp2f(sm[w] - ref);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v = 0.0f;
    for (int w = 0; w < 4; ++w) v += so[w][lane + 64 * i] * __builtin_amdgcn_exp2f(sm[w] - ref);
    const float y = total > 0.0f ? v / total : (total == 0.0f ? 0.0f : total);
    p.O[s * p.ld_o + int64_t(h) * D + lane + 64 * i] = uint16_t(pack_bf16x2(y, y));
  }
  if (lane == 0 && p.lse) p.lse[s * p.H + h] = total == 0.0f ? NEG_INF : ref + __builtin_amdgcn_logf(total);
}

}  // namespace

size_t attn_decode_ws(int64_t n_seq, int H, int H_kv, int d, int64_t max_pages, int page_len) { return 0; }

hipError_t launch_attn_decode(const AttnDecodeLaunch& p, hipStream_t st) {
  const dim3 grid{unsigned(p.c.n_seq * p.H)};
  if (p.c.d == 128)
    attn_decode_kernel<128><<<grid, 256, 0, st>>>(p);
  else
    attn_decode_kernel<64><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace uq
