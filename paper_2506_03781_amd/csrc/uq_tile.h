// Device helpers of attentions whose rows lie in LDS as tiles of 32 rows of 128
// bf16: their swizzled layout, copies into it, and the operands of
// v_mfma_f32_32x32x16_bf16 out of it.  gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace uq {

namespace {

typedef __bf16 bf16x8a __attribute__((ext_vector_type(8)));
typedef float f32x16a __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4a __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2a __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void_a;
typedef const __attribute__((address_space(1))) void glb_void_a;

constexpr int D = 128;                       // head dimension
constexpr int NB = 32;                       // rows (keys or queries) per tile
constexpr int TILE16 = NB * D * 2 / 16;      // 16-byte slots of a tile (512)
constexpr float LOG2E = 1.44269504088896341f;

__device__ __forceinline__ f32x16a mfma(const bf16x8a& a, const bf16x8a& b, const f32x16a& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float exp2a(float x) { return __builtin_amdgcn_exp2f(x); }

// bf16 value nearest to x (ties to even), as fp32.
__device__ __forceinline__ float bf16_round(float x) { return float(__bf16(x)); }

// Tile row held by accumulator slot r of this lane (rows read in perm32 order).
__device__ __forceinline__ int slot_row(int r, int lane) { return 16 * (r >> 3) + 8 * (lane >> 5) + (r & 7); }

// Swap bits 2 and 3 of a row index below 32 (an involution).
__device__ __forceinline__ int perm32(int r) { return (r & 19) | ((r & 4) << 1) | ((r >> 1) & 4); }

template <int N>
__device__ __forceinline__ void vm_wait() {
  // s_waitcnt fields: vmcnt[3:0] and [15:14], expcnt[6:4], lgkmcnt[11:8]
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// Wait until at most `ahead` (0..2) later tiles of PW copies each are in flight.
template <int PW>
__device__ __forceinline__ void wait_tiles(int ahead) {
  if (ahead >= 2) vm_wait<2 * PW>();
  else if (ahead == 1) vm_wait<PW>();
  else vm_wait<0>();
}

__device__ __forceinline__ void lds_wait_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): this wave's LDS reads are done
  __builtin_amdgcn_s_barrier();
}

// Chunk swizzle of tile row rho: the two 2-bit fields of rho % 16 swapped.
// It is a bijection on rho % 16, so the 16 rows a quarter-wavefront reads at
// one chunk fall in 16 distinct slots, and four consecutive rows differ in
// bits 2-3, so the two adjacent chunks of four consecutive rows that a
// transpose read takes also fall in 8 distinct slots.
__device__ __forceinline__ int swz(int rho) { return ((rho & 3) << 2) | ((rho >> 2) & 3); }

// Row tile (32 rows of 128 bf16 = 512 slots of 16 bytes): slot s holds chunk
// (s % 16) ^ swz(rho) of tile row rho = s / 16, and tile row rho holds
// source row perm32(rho) of the tile.  Copy block blk fills slots 64 blk ..
// + 64; row_off is this lane's byte offset in the source tile for block blk.
__device__ __forceinline__ uint32_t row_off(int blk, int lane, int ld = D) {
  const int s = blk * 64 + lane;
  const int rho = s >> 4, c = (s & 15) ^ swz(rho);
  return uint32_t(perm32(rho)) * uint32_t(ld) * 2u + uint32_t(c * 16);
}

// A copy of 64 slots: lane l's 16 bytes at base + off land in slot l of dst.
__device__ __forceinline__ void copy16(const void* base, uint32_t off, u32x4a* dst) {
  __builtin_amdgcn_global_load_lds((glb_void_a*)(static_cast<const char*>(base) + off), (lds_void_a*)dst, 16, 0, 0);
}

// A or B fragment of k-step j (d = 16 j + 8 (lane / 32) .. + 8) of tile row lane % 32.
__device__ __forceinline__ bf16x8a row_frag(const u32x4a* tile, int j, int lane) {
  const int rho = lane & 31, c = 2 * j + (lane >> 5);
  return __builtin_bit_cast(bf16x8a, tile[rho * 16 + (c ^ swz(rho))]);
}

typedef short v4i16a __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16a lds_v4i16a;

// A fragment of the transposed row tile: rows d = 32 db .. + 32 over the 16
// tile rows (keys or queries, in source order) of half h; lane supplies
// d = 32 db + lane % 32 and source rows 16 h + 8 (lane / 32) .. + 8.
// ds_read_b64_tr_b16 gives lane i of each 16-lane group, in slot j, element
// i % 4 of the 8 bytes addressed by lane 4 j + i / 4 of the group; lane
// 4 j + q addresses source row r0 + j, columns d0 + 4 q .. + 3, so lane i
// receives column d0 + i of rows r0 .. r0 + 3: half the fragment.
__device__ __forceinline__ bf16x8a col_frag(const u32x4a* tile, int db, int h, int lane) {
  const int g = lane >> 4, i = lane & 15;
  const int d = 32 * db + 16 * (g & 1) + 4 * (i & 3);
  const char* base = reinterpret_cast<const char*>(tile);
  v4i16a part[2];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const int rho = perm32(16 * h + 8 * (g >> 1) + 4 * hh + (i >> 2));
    const int off = rho * D * 2 + (((d >> 3) ^ swz(rho)) << 4) + ((d & 7) >> 2) * 8;
    part[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16a*)(base + off));
  }
  return __builtin_bit_cast(bf16x8a, part);
}

// row_frag and col_frag for a loop over tiles of one array of stages (256-byte aligned): a lane's addresses
// differ from its first one in single bits and in constants, which are the reads' own, so that a read costs
// one instruction for its address in place of three.  `bytes`: of the tile in the stage, a constant.
typedef __attribute__((address_space(3))) u32x4a lds_u32x4a;
struct LaneTile {
  uint32_t r, c;  // of k-step 0; of d block 0, half 0

  __device__ __forceinline__ LaneTile(const u32x4a* smem, int lane) {
    const uint32_t at = uint32_t(reinterpret_cast<uintptr_t>((lds_void_a*)smem));
    const int i = lane & 15, g = lane >> 4, rho = 4 * (g >> 1) + (i >> 2);
    r = at + uint32_t((lane & 31) * 256 + (((lane >> 5) ^ swz(lane & 31)) << 4));
    c = at + uint32_t(rho * 256 + (((2 * (g & 1) + ((i & 3) >> 1)) ^ swz(rho)) << 4) + (i & 1) * 8);
  }
  // Of the stage that begins `bytes` behind the first one (opaque: 16 addresses are not held across the loop).
  __device__ __forceinline__ LaneTile at(uint32_t bytes) const {
    LaneTile t = *this;
    t.r += bytes;
    t.c += bytes;
    asm volatile("" : "+v"(t.r), "+v"(t.c));
    return t;
  }
  __device__ __forceinline__ bf16x8a row(int j, uint32_t bytes) const {
    return __builtin_bit_cast(bf16x8a, *reinterpret_cast<const lds_u32x4a*>(uintptr_t((r ^ uint32_t(j << 5)) + bytes)));
  }
  __device__ __forceinline__ bf16x8a col(int db, int h, uint32_t bytes) const {
    v4i16a part[2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
      part[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<lds_v4i16a*>(uintptr_t((c ^ uint32_t(hh << 5 | db << 6)) + (bytes + h * 4096 + hh * 2048))));
    return __builtin_bit_cast(bf16x8a, part);
  }
};

// Slots 8 h .. 8 h + 7 as a bf16 B operand.
__device__ __forceinline__ bf16x8a pack_half(const float (&v)[16], int h) {
  bf16x8a w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = __bf16(v[8 * h + i]);
  return w;
}

__device__ __forceinline__ f32x16a zero16() {
  f32x16a z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
  return z;
}

}  // namespace

}  // namespace uq
