// lds_loads.h -- helpers of the decode kernels whose rows go from memory straight
// into a wavefront's own part of LDS (gfx950).
#pragma once

#include "decode_split.h"

namespace hwkv {
namespace {

// 16 bytes (4 with DWORD) per lane from a buffer into LDS, at 16 (4) x lane of
// lds_block; past the descriptor's range zeros arrive.  The load has no
// destination register, and the kernel waits for it itself (wait_loads): as a
// builtin it would make the compiler wait for every load in flight before each
// LDS read.
template <bool DWORD>
__device__ __forceinline__ void stage_lds(__amdgpu_buffer_rsrc_t r, uint32_t lds_block, int voffset,
                                          int soffset) {
  if constexpr (DWORD)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen nt lds" ::"s"(lds_block),
                 "v"(voffset), "s"(r), "s"(soffset)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds" ::"s"(lds_block),
                 "v"(voffset), "s"(r), "s"(soffset)
                 : "memory", "m0");
}

// No vector memory operation of the wave is in flight.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The largest over lanes l16, l16 + 16, l16 + 32, l16 + 48.
__device__ __forceinline__ float max_of_rows(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t y = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Two bf16 of the signed bytes E of two words, low first (exact).
template <int E>
__device__ __forceinline__ uint32_t codes_bf16x2(uint32_t x, uint32_t y) {
  const f32x2_t f = {(float)(int)(int8_t)(x >> (8 * E)), (float)(int)(int8_t)(y >> (8 * E))};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

}  // namespace
}  // namespace hwkv
