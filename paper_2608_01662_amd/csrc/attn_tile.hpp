// Pieces of the attention kernels: the tile of latent rows in LDS, transposed reads, the online softmax's
// constants. (The layouts' reasons are given where the kernels use them.)
#pragma once
#include "device.hpp"

namespace lsa {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLazy = 8.0f;  // rescale when the max grows by more than this (log2 units)

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// V^T operand of a product over tokens from token-major LDS: two transposed reads of 4 tokens each.
__device__ __forceinline__ u32x4 tr16_pair(const uint8_t* pa, const uint8_t* pb) {
  const s16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(pa));
  const s16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(pb));
  const u32x2 a2 = __builtin_bit_cast(u32x2, va), b2 = __builtin_bit_cast(u32x2, vb);
  return u32x4{a2.x, a2.y, b2.x, b2.y};
}

constexpr int kMlaT = 32;
constexpr int kMlaTile = 36 * 1024;  // 72 chunks x 32 tokens x 16 bytes
constexpr int kMlaBufs = 3;          // tile buffers: scored, in the value products, loading
constexpr int kMlaLoads = 9;         // direct loads per value wave per tile (36 x 1 KB)
constexpr int kMlaPHead = 80;        // bytes per head in a P slot: 32 bf16 tokens + 16 B of padding
constexpr int kMlaPSlot = 64 * kMlaPHead + 2 * 64 * 4;  // per tile parity: P of 64 heads + the reference maxima of both token halves
__device__ __forceinline__ int mla_swz(int o, int j) { return ((j & 2) << 1) | ((j & 4) >> 1) | (o & 1); }
constexpr int kMlaHalf = 18 * 1024;  // the second 16 tokens of a tile start 18 blocks later
// Nine direct loads of one 1152-byte row piece per lane: load k reads the 16 bytes at src + 128 k
// and writes LDS bytes [lds + 1024 k + 16 lane, +16). The loads share one address and carry
// 128 k as their immediate offset, which these loads add to the LDS address as well, so M0 steps
// by 1024 - 128 per load. Written as one asm block so that the compiler does not see LDS being
// written by vector-memory loads: it would otherwise drain every such load in flight before any
// later LDS read it cannot prove disjoint; callers order the loads with explicit vmcnt waits and
// barriers. M0, which holds the LDS address of the loads, is saved and restored; the s_nop after
// each write of M0 is the wait state before a load may read it.
__device__ __forceinline__ void lds_dma_row9(const uint8_t* src, uint32_t lds) {
  uint32_t save;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:128\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:256\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:384\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:512\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:640\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:768\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:896\n\t"
      "s_add_u32 m0, m0, 0x380\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off offset:1024\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(save)
      : "v"(src), "s"(lds)
      : "memory", "scc");
}

// The maxima of x and of y over the four 16-lane rows (lanes l, l ^ 16, l ^ 32, l ^ 48), sharing
// the lane swaps: the first swap leaves rows (x0, y0, x2, y2) and (x1, y1, x3, y3), the second
// (row halves) rows x, y, x, y of the full maxima, the last hands each lane both.
__device__ __forceinline__ void max4_xor16_32_pair(float& x, float& y) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  const float z = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(z), __float_as_uint(z), false, false);
  const float w = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
  const auto c = __builtin_amdgcn_permlane16_swap(__float_as_uint(w), __float_as_uint(w), false, false);
  x = __uint_as_float(c[0]);
  y = __uint_as_float(c[1]);
}
constexpr float kNoRef = -3.40282347e38f;  // reference maximum before a head's first score (finite, so
                                           // exp2(s - m) needs no guard: masked scores are -inf)

// eight bf16 scaled by f (rounded to nearest even again)
__device__ __forceinline__ u32x4 scale_bf16x8(u32x4 v, float f) {
  u32x4 r;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    r[k] = pack_bf16x2(__uint_as_float(v[k] << 16) * f, __uint_as_float(v[k] & 0xFFFF0000u) * f);
  return r;
}

__device__ __forceinline__ f32x4 bf16x4_f32(u32x2 v) {
  return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
               __uint_as_float(v.y & 0xFFFF0000u)};
}

}  // namespace lsa
