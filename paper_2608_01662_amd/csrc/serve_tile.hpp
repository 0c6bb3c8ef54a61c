// What the attention kernels over whole contexts share: wave-wide scans, direct loads of cache rows, fp8 codes as bf16.
#pragma once
#include "device.hpp"

namespace lsa {

// What loads of positions that nobody attends to read instead (behind the context, in unmapped pages): zeros,
// since a weight of zero does not silence a NaN or an infinity in V.
static __device__ __attribute__((aligned(256))) const uint8_t zero_row[1152] = {};

// (a wave-uniform value that the compiler cannot know to be: kept in a scalar register)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8: within rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15: rows 0 and 2 into 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31: row 1 into 2 and 3
  return x;
}

// ---------------------------------------------------------------- direct global -> LDS loads
// 16 (4) bytes per lane from `src` to LDS bytes lds + 16 (4) lane. The compiler does not see these loads, so
// that it does not drain them before every LDS read; callers wait with explicit vmcnt counts. M0 holds the LDS
// address and is restored; the s_nop is the wait state before a load may read it.
__device__ __forceinline__ void lds_dma16(const uint8_t* src, uint32_t lds) {
  uint32_t save;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
               : "=&s"(save) : "v"(src), "s"(lds) : "memory");
}
__device__ __forceinline__ void lds_dma4(const uint8_t* src, uint32_t lds) {
  uint32_t save;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
               : "=&s"(save) : "v"(src), "s"(lds) : "memory");
}


// eight e4m3 codes -> eight bf16 (exact)
__device__ __forceinline__ u32x4 fp8x8_bf16(uint32_t lo, uint32_t hi) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true))};
}

}  // namespace lsa
